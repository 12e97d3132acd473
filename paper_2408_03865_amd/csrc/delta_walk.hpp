// delta_walk.hpp -- the walks of the gated delta rule over the chunks of a row.
//
// For every head, with S' = a_t S_{t-1} (a_t = exp(g_t), 0 at a sequence start):
//   e_t = v_t - S'^T k_t,  u_t = beta_t e_t,  S_t = S' + k_t u_t^T,  out_t = scale S_t^T q_t.
// In chunks of 64 tokens, with what delta_prep.hip made of the keys and queries (H, P) and the weights in, up
// and A of linear_walk.hpp:
//   x = v - in (K^T S),  e = x - H (beta x),  u = beta e
//   out = scale in (Q^T S) + P u,      S <- A S + K (up u)
// and backwards in time, D the gradient of the state that leaves the chunk, dx_t that of u_t:
//   x = up (K^T D) + P^T dout,  du = x - H^T (beta x),  dv = beta du
//   D <- A D + scale Q (in dout) - K (in dv)
// The gradients of beta are du . e, those of the log decays sums of out . dout - v . dv over the tokens that
// follow in the sequence, up to a boundary, plus the product of S and D there: with F the gradient of S',
// dg_t = <F_t, S'_t> = <D_t, S_t> - v_t . dv_t (S_t - beta_t k_t v_t^T is linear in a_t), and the <D, S> of
// the token before is dg_t + out . dout there.
//
// Mapping.  The columns of S (v's features) need nothing of each other: each wave owns 16 of them and all of
// k's features, in registers, in the layout that an MFMA result has and, four rows of it a lane, an MFMA operand
// takes.  So do x, e, u and the outs: four consecutive tokens of a feature a lane.  A block's waves share the chunk's
// K, Q, H and P in LDS, which the next chunk's loads pass through registers.
// bf16: what is no input is split into three bf16 terms, all 24 bits of it: the state, H, P, x and u.  Outs and errors are
// small differences of their terms where keys are near each other, and of large ones where a token replaces what the
// state held: with two terms outs behind a value 100 times the others, which the next token of its key replaces, were 2.1e-2
// off in the 2-norm and not 1.7e-3 (8 x 4096 tokens, 32 heads of 128 x 128 took 506 us and not 620).
//
// What bounds them: the instructions of two waves a SIMD.  8 x 32 rows of 128 features are 2048 waves, two for each of 1024 SIMDs; with
// more rows the registers, 190 to 245 a wave, would leave room for no more.  In the backward also the memory that they keep states and
// errors in.  8 x 4096 tokens, 32 heads of 128 x 128, bf16, in cycles that a unit works and bytes moved:
//   outs    570 us   VALU 59%, matrix 47%, LDS 25%; 1.16 GB, 2.0 TB/s
//   states  745 us   VALU 45%, matrix 32%, LDS 17%; 2.79 GB, 3.7 TB/s
//   reverse 967 us   VALU 41%, matrix 21%, LDS 17%; 4.40 GB, 4.6 TB/s
// Nearly half of the VALU work is splitting of states, errors and products.
//
// Infinities and NaN: a chunk whose k or q holds one, or whose u (du) a wave finds one in, is walked by that wave token
// by token from the definition, so that 0 times it reaches no other token or sequence.  A state that holds one makes x
// and with it u such, whatever the weights, 0 among them.
#pragma once

#include "linear_walk.hpp"
#include "delta.hpp"

namespace pm {

enum DeltaMode : int { kDeltaOut = 0, kDeltaSum = 1, kDeltaStates = 2 };

// A chunk's operands.
template <typename T, int KC, int NH, int NP, bool Q>
struct DeltaTiles {
    using Frag = typename Mat<T>::Frag;
    __attribute__((aligned(16))) T k[KC * kC];
    __attribute__((aligned(16))) T q[Q ? KC * kC : 8];
    __attribute__((aligned(16))) Frag h[NH][kDeltaTiles][64];
    __attribute__((aligned(16))) Frag p[NP ? NP : 1][NP ? kDeltaTiles : 1][64];
    __attribute__((aligned(16))) float coef[3][kC];
    __attribute__((aligned(16))) float misc[4];
};
// Two of them, the next chunk's written during this one with one barrier a chunk and not two, for blocks of four waves where a CU
// holds two blocks all the same: those are the segments' sums in time, which have no P.  Us of calls with one and with two: backward
// of 4 x 24 heads x 2048, 64 x 64, 371, 358; 30001 tokens forward, 24 heads of 128 x 64, 695, 690.
template <typename T, int KC, int VP, int NH, int NP, bool Q>
constexpr int delta_buffers() {
    return VP == 64 && (int)sizeof(DeltaTiles<T, KC, NH, NP, Q>) * 2 <= 78 * 1024 ? 2 : 1;
}
template <typename T, int KC, int VP, int NH, int NP, bool Q, int DOTS>
struct DeltaSmem {
    static constexpr int kBuffers = delta_buffers<T, KC, VP, NH, NP, Q>();
    DeltaTiles<T, KC, NH, NP, Q> b[kBuffers];
    __attribute__((aligned(16))) float dot[2][DOTS ? DOTS : 1][VP / 16][kC];
    float xdot[2][VP / 16];
};

__host__ __device__ constexpr int delta_tile(int i, int j) { return i * (i + 1) / 2 + j; }

// The prepared products on their way into LDS, H in NH terms and, unless NP is 0, P in NP.
template <typename T, int NH, int NP, int THREADS>
struct ProductRegs {
    using M = Mat<T>;
    using Frag = typename M::Frag;
    static constexpr int kOne = (int)kDeltaProduct / 4, kVecs = (NP ? 2 : 1) * kOne, kPasses = (kVecs + THREADS - 1) / THREADS;
    f32x4 w[kPasses];
    __device__ void load(int tid, const float* p, int64_t unit) {
        const f32x4* v = reinterpret_cast<const f32x4*>(p) + unit * (2 * kOne);
#pragma unroll
        for (int i = 0; i < kPasses; ++i) w[i] = v[min(i * THREADS + tid, kVecs - 1)];
    }
    template <int N>
    __device__ static void put(const f32x4& v, Frag* to) {
        Frag f[N];
        M::template split<N>(v, f);
#pragma unroll
        for (int n = 0; n < N; ++n) to[n * kOne] = f[n];
    }
    __device__ void store(int tid, Frag* h, Frag* p) const {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {             // a wave's lanes have one tile
            const int at = i * THREADS + tid;
            if ((i + 1) * THREADS <= kOne || __builtin_amdgcn_readfirstlane(at) < kOne) {
                put<NH>(w[i], h + at);
            } else if constexpr (NP != 0) {
                if (kVecs % THREADS == 0 || __builtin_amdgcn_readfirstlane(at) < kVecs) put<NP>(w[i], p + (at - kOne));
            }
        }
    }
};

// K's or Q's chunk on its way into LDS: as TileRegs, with one address a vector whatever the head's features are, so that no branch
// stands between the loads and the products that they run under.
template <typename T, int ROWS, int THREADS>
struct FeatureRegs : TileRegs<T, ROWS, THREADS> {
    using Base = TileRegs<T, ROWS, THREADS>;
    __device__ void load(int tid, const T* p, int rows, int t0, int L) {
        typedef const __attribute__((address_space(1))) char* Bytes;
        typedef const __attribute__((address_space(1))) typename Storage<T>::Vec* Global;
        const bool tiny = L < Base::kPer;               // rows shorter than a vector: settle() reads them
        const Bytes base = (Bytes)(uintptr_t)(tiny ? reinterpret_cast<const T*>(&walk_zero) : p);
        const uint32_t tok = tiny ? 0u : (uint32_t)min(t0 + (tid % Base::kLanes) * Base::kPer, L - Base::kPer), step = tiny ? 0u : (uint32_t)L;
#pragma unroll
        for (int i = 0; i < Base::kPasses; ++i) {
            const uint32_t row = (uint32_t)min(tid / Base::kLanes + i * Base::kRowsPass, rows - 1);
            Base::w[i] = *(Global)(base + (row * step + tok) * (uint32_t)sizeof(T));
        }
    }
};

// A chunk of one feature's row, as a lane's result registers hold it: tokens 16 i + 4 (lane / 16) .. + 3 of row lane % 16, for the
// four tiles i.  In bf16 those are 8 bytes each; 16-byte vectors of memory serve two tiles, whose halves the lanes of
// neighbouring rows of 16 swap, so that a row's bytes move in pieces of 64 and not of 32.
template <typename T>
struct TokenRegs {
    using Frag = typename Mat<T>::Frag;
    static constexpr bool kPairs = sizeof(T) == 2;
    static constexpr int kVecs = kPairs ? 2 : 4, kPer = Storage<T>::kPerVec;
    u32x4 w[kVecs];

    // a vector's first token
    __device__ static int at(int l, int i) {
        return kPairs ? i * 32 + ((l >> 4) & 1) * 16 + (l >> 5) * 8 : i * 16 + (l >> 4) * 4;
    }
    // p: the feature's row, t0: the chunk's first token
    __device__ void load(const T* p, int64_t t0, int l, int64_t L) {
        if (t0 + kC <= L) {
#pragma unroll
            for (int i = 0; i < kVecs; ++i) w[i] = load_vec<T, kPer>(p + t0 + at(l, i));
        } else {
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                float v[kPer];
#pragma unroll
                for (int r = 0; r < kPer; ++r) {
                    const int64_t t = t0 + at(l, i) + r;
                    v[r] = t < L ? Storage<T>::load1(p + t) : 0.0f;
                }
                w[i] = Storage<T>::pack(v);
            }
        }
    }
    __device__ void store(T* p, int64_t t0, int l, int64_t L) const {
        if (t0 + kC <= L) {
#pragma unroll
            for (int i = 0; i < kVecs; ++i) *reinterpret_cast<typename Storage<T>::Vec*>(p + t0 + at(l, i)) = w[i];
        } else {
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                float v[kPer];
                Storage<T>::unpack(w[i], v);
#pragma unroll
                for (int r = 0; r < kPer; ++r)
                    if (t0 + at(l, i) + r < L) Storage<T>::store1(p + t0 + at(l, i) + r, v[r]);     // of this type already
            }
        }
    }
    __device__ static void swap(uint32_t& a, uint32_t& b) {      // a's odd rows of 16 lanes with b's even ones
        const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
        a = r[0];
        b = r[1];
    }
    // the tiles' values; mask: all ones, or 0 for a row that the tensor lacks
    __device__ void get(uint32_t mask, Frag (&f)[4]) const {
        if constexpr (kPairs) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                u32x4 v = w[i] & mask;
                uint32_t a = v.x, b = v.y, c = v.z, d = v.w;
                swap(a, c);
                swap(b, d);
                f[2 * i] = Frag{a, b};
                f[2 * i + 1] = Frag{c, d};
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[i] = __builtin_bit_cast(f32x4, u32x4(w[i] & mask));
        }
    }
    __device__ void set(const f32x4 (&v)[4]) {
        if constexpr (kPairs) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u32x2 x = Mat<T>::round(v[2 * i]), y = Mat<T>::round(v[2 * i + 1]);
                uint32_t a = x.x, b = x.y, c = y.x, d = y.y;
                swap(a, c);
                swap(b, d);
                w[i] = u32x4{a, b, c, d};
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(u32x4, v[i]);
        }
    }
};

// What a value's pattern of 32 bits is over that of its bf16 rounding (as 32 bits): 16 bits, a signed number; where a tie went down
// one less.
__device__ __forceinline__ uint32_t rest_of(float v, uint32_t rounded) {
    return (uint32_t)max(min((int32_t)(__float_as_uint(v) - rounded), 0x7fff), -0x8000) & 0xffffu;
}

// 16 bits a token that are no numbers, as TokenRegs has a row's bf16.
struct HalfRegs : TokenRegs<bf16_t> {
    __device__ void load(const uint16_t* p, int64_t t0, int l, int64_t L) {
        if (t0 + kC <= L) {
            TokenRegs::load(reinterpret_cast<const bf16_t*>(p), t0, l, L);
        } else {
#pragma unroll
            for (int i = 0; i < kVecs; ++i)
#pragma unroll
                for (int r = 0; r < kPer; r += 2) {
                    const int64_t t = t0 + at(l, i) + r;
                    w[i][r / 2] = (t < L ? p[t] : 0u) | (uint32_t)(t + 1 < L ? p[t + 1] : 0u) << 16;
                }
        }
    }
    // what TokenRegs<bf16_t>::set() leaves of the values
    __device__ void set_rest(const f32x4 (&v)[4]) {
        const auto pair = [](float x, float y, uint32_t rounded) { return rest_of(x, rounded << 16) | rest_of(y, rounded & 0xffff0000u) << 16; };
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x4 &x = v[2 * i], &y = v[2 * i + 1];
            const u32x2 xr = Mat<bf16_t>::round(x), yr = Mat<bf16_t>::round(y);
            uint32_t a = pair(x.x, x.y, xr.x), b = pair(x.z, x.w, xr.y), c = pair(y.x, y.y, yr.x), d = pair(y.z, y.w, yr.y);
            swap(a, c);
            swap(b, d);
            w[i] = u32x4{a, b, c, d};
        }
    }
    __device__ void store(uint16_t* p, int64_t t0, int l, int64_t L) const {
        if (t0 + kC <= L) {
            TokenRegs::store(reinterpret_cast<bf16_t*>(p), t0, l, L);
        } else {
#pragma unroll
            for (int i = 0; i < kVecs; ++i)
#pragma unroll
                for (int r = 0; r < kPer; ++r) {
                    const int64_t t = t0 + at(l, i) + r;
                    if (t < L) p[t] = (uint16_t)(w[i][r / 2] >> (r % 2 * 16));
                }
        }
    }
};

// Errors whole in 32 bits: as bf16, rounded half up, which the products take, and the lower halves of the fp32 patterns, which
// make up the rest: a pattern is the rounded one's plus its own lower half, taken for a signed number.
__device__ __forceinline__ uint32_t halves(uint32_t a, uint32_t b, bool upper) {     // of b and a, b's above
    return __builtin_amdgcn_perm(b, a, upper ? 0x07060302u : 0x05040100u);
}
// one of a pair of them
__device__ __forceinline__ float whole(uint32_t hi, uint32_t lo, int which) {
    return __uint_as_float(which ? (hi & 0xffff0000u) + (uint32_t)((int32_t)lo >> 16) : (hi << 16) + (uint32_t)((int32_t)(lo << 16) >> 16));
}
template <typename T>
struct ErrorRegs {
    TokenRegs<T> hi;
    HalfRegs lo;
    __device__ void set(const f32x4 (&e)[4]) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const u32x4 x = __builtin_bit_cast(u32x4, e[2 * i]), y = __builtin_bit_cast(u32x4, e[2 * i + 1]);
                const u32x4 xr = x + 0x8000u, yr = y + 0x8000u;
                const auto pairs = [](const u32x4& x, const u32x4& y, bool upper) {
                    uint32_t a = halves(x.x, x.y, upper), b = halves(x.z, x.w, upper), c = halves(y.x, y.y, upper), d = halves(y.z, y.w, upper);
                    TokenRegs<T>::swap(a, c);
                    TokenRegs<T>::swap(b, d);
                    return u32x4{a, b, c, d};
                };
                hi.w[i] = pairs(xr, yr, true);
                lo.w[i] = pairs(x, y, false);
            }
        } else {
            hi.set(e);
        }
    }
    __device__ void get(uint32_t mask, f32x4 (&e)[4]) const {
        typename Mat<T>::Frag f[4];
        hi.get(mask, f);
        if constexpr (sizeof(T) == 2) {
            Mat<bf16_t>::Frag h[4];
            lo.get(mask, h);
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = f32x4{whole(f[i].x, h[i].x, 0), whole(f[i].x, h[i].x, 1), whole(f[i].y, h[i].y, 0), whole(f[i].y, h[i].y, 1)};
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = f[i];
        }
    }
    __device__ void store(T* row, uint16_t* low, int64_t t0, int l, int64_t L) const {
        hi.store(row, t0, l, L);
        if constexpr (sizeof(T) == 2) lo.store(low, t0, l, L);
    }
    __device__ void load(const T* row, const uint16_t* low, int64_t t0, int l, int64_t L) {
        hi.load(row, t0, l, L);
        if constexpr (sizeof(T) == 2) lo.load(low, t0, l, L);
    }
    // one token's
    __device__ static void put(T* at, uint16_t* low, float e) {
        if constexpr (sizeof(T) == 2) {
            at->bits = (uint16_t)((__float_as_uint(e) + 0x8000u) >> 16);
            *low = (uint16_t)__float_as_uint(e);
        } else {
            *at = e;
        }
    }
    __device__ static float take(const T* at, const uint16_t* low) {
        if constexpr (sizeof(T) == 2) return whole(at->bits, *low, 0);
        else return *at;
    }
};

// v at four consecutive tokens t.. of a row
template <typename TO>
__device__ __forceinline__ void store_tokens(TO* row, int64_t t, int64_t L, const f32x4& v) {
    if (t + 4 <= L) {
        if constexpr (sizeof(TO) == 2) *reinterpret_cast<u32x2_a2*>(row + t) = Mat<bf16_t>::round(v);
        else *reinterpret_cast<u32x4_a4*>(row + t) = __builtin_bit_cast(u32x4, v);
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (t + r < L) Storage<TO>::store1(row + t + r, v[r]);
    }
}

// States of a row that the backward keeps: those before its chunks, and in bf16 the last one, in place of `bound`.
template <typename T>
__host__ __device__ constexpr int delta_slots(int chunks) { return Mat<T>::kSplit ? chunks + 1 : chunks; }

// The state: rows 16 k + 4 (lane / 16) .. + 3, column lane % 16 of the wave's 16.
template <int KF>
struct DeltaState {
    f32x4 s[KF];
    template <typename F>
    __device__ void each(F f) {
        const int l = here(lane_id());
#pragma unroll
        for (int k = 0; k < KF; ++k) f(k * 16 + (l >> 4) * 4, l & 15, s[k]);
    }
    // rows x cols, row-major with `stride`; zf: the wave's first column
    __device__ void load(const float* p, int rows, int cols, int zf, int stride) {
        each([&](int x, int z, f32x4& v) {
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = p && x + r < rows && zf + z < cols ? p[(int64_t)(x + r) * stride + zf + z] : 0.0f;
        });
    }
    __device__ void store(float* p, int rows, int cols, int zf, int stride) {
        each([&](int x, int z, f32x4& v) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (x + r < rows && zf + z < cols) p[(int64_t)(x + r) * stride + zf + z] = v[r];
        });
    }
    // columns of the identity of `rows` from zf on: ones of rows that no key has would only be decayed, where decays are above 0 to
    // infinities, whose products with the 0 that the state holds there are none
    __device__ void identity(int zf, int rows) {
        each([&](int x, int z, f32x4& v) {
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = x + r == zf + z && x + r < rows ? 1.0f : 0.0f;
        });
    }
    __device__ void decay(float a) {
#pragma unroll
        for (int k = 0; k < KF; ++k) s[k] *= a;
    }
    __device__ void clear() {
#pragma unroll
        for (int k = 0; k < KF; ++k) s[k] = f32x4{0, 0, 0, 0};
    }
    // transposed: column z is a row of KF * 16
    __device__ void keep(float* p, int zf) {
        each([&](int x, int z, f32x4& v) { *reinterpret_cast<f32x4*>(p + (zf + z) * (KF * 16) + x) = v; });
    }
    // the sum of the products with what keep() left
    __device__ float dot_kept(const float* p, int zf) {
        float d = 0.0f;
        each([&](int x, int z, f32x4& v) {
            const f32x4 o = *reinterpret_cast<const f32x4*>(p + (zf + z) * (KF * 16) + x);
#pragma unroll
            for (int r = 0; r < 4; ++r) d = fmaf(o[r], v[r], d);
        });
        return d;
    }
    // one token, of which column j of a tile is the key's or query's: sum over the rows of it times the column.  absent: a row that it
    // has 0 of is not met, also where the state is infinite there
    template <typename T>
    __device__ float against(const T* tile, int j, bool absent = false) {
        const int l = here(lane_id());
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < KF; ++k) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float x = tile_value(tile + k * 16 * kC, (l >> 4) * 4 + r, j);
                v = absent && x == 0.0f ? v : fmaf(x, s[k][r], v);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        v += __shfl_xor(v, 16);
        v += __shfl_xor(v, 32);
        return v;
    }
    template <typename T>
    __device__ void add(const T* tile, int j, float f) {
        const int l = here(lane_id());
#pragma unroll
        for (int k = 0; k < KF; ++k) {
#pragma unroll
            for (int r = 0; r < 4; ++r) s[k][r] = fmaf(tile_value(tile + k * 16 * kC, (l >> 4) * 4 + r, j), f, s[k][r]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// A read that stays by itself: two of them in one instruction leave the halves of two operands side by side, and moves to part
// them cost more than the instruction.
template <typename F>
__device__ __forceinline__ F alone(const F* p) {
    return *(const volatile __attribute__((address_space(3))) F*)p;
}

// A tile of a product as an operand, or turned: rows 4 (lane / 16) .. + 3 of it, column lane % 16.
template <typename T, bool TURNED>
__device__ __forceinline__ typename Mat<T>::Frag product_tile(int l, const typename Mat<T>::Frag* tile) {
    using Frag = typename Mat<T>::Frag;
    if constexpr (!TURNED) {
        return alone(tile + l);
    } else if constexpr (sizeof(T) == 2) {
        const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(const_cast<Frag*>(tile + (l & 3) * 16 + (l >> 4) * 4 + ((l & 15) >> 2))));
        return __builtin_bit_cast(u32x2, v);
    } else {
        const float* p = reinterpret_cast<const float*>(tile + ((l & 15) >> 2) * 16 + (l >> 4) * 4) + (l & 3);
        return Frag{p[0], p[4], p[8], p[12]};
    }
}

// acc[i] (token tile i) += product tiles (i, j) times y[j], over j <= i, or with REV over j >= i of the turned tiles.  The tiles'
// chains take turns: a matrix instruction that takes the result of the one before waits for it.
template <typename T, bool REV, int NA, int NB>
__device__ __forceinline__ void multiply_product(int lane, const typename Mat<T>::Frag (*tiles)[kDeltaTiles][64],
                                                 const typename Mat<T>::Frag (&y)[4][NB], f32x4 (&acc)[4]) {
    using Frag = typename Mat<T>::Frag;
    const int l = here(lane);
#pragma unroll
    for (int jp = 0; jp < 2; ++jp) {
        __builtin_amdgcn_sched_barrier(0);
        const auto in = [&](int i, int j) { return REV ? j >= i : j <= i; };
        const auto at = [&](int i, int j) { return REV ? delta_tile(j, i) : delta_tile(i, j); };
#pragma unroll
        for (int n = NA - 1; n >= 0; --n) {              // terms' products below the last term's size are left out
            Frag f[4][2];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int q = 0; q < 2; ++q) f[i][q] = in(i, 2 * jp + q) ? product_tile<T, REV>(l, tiles[n][at(i, 2 * jp + q)]) : Frag{};
#pragma unroll
            for (int m = NB - 1; m >= 0; --m) {
                if (n + m >= (NA > NB ? NA : NB)) continue;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (in(i, 2 * jp) || in(i, 2 * jp + 1)) acc[i] = Mat<T>::mma(f[i][0], f[i][1], y[2 * jp][m], y[2 * jp + 1][m], acc[i]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// S += rows of a tile times w, over the chunk's tokens; few: only the state's first 32 rows are any
template <typename T, int KF, int NS>
__device__ __forceinline__ void add_tokens(int lane, DeltaState<KF>& S, const T* tile, const typename Mat<T>::Frag (&w)[4][NS], bool few) {
    using M = Mat<T>;
    const int l = here(lane);
    if (few) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            typename M::Frag y[2][2];
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    y[q][h] = alone(reinterpret_cast<const typename M::Frag*>(tile + q * 16 * kC + M::direct_at(l, 2 * p + h)));
#pragma unroll
            for (int n = NS - 1; n >= 0; --n)
#pragma unroll
                for (int q = 0; q < 2; ++q) S.s[q] = M::mma(y[q][0], y[q][1], w[2 * p][n], w[2 * p + 1][n], S.s[q]);
        }
        return;
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int k = 0; k < KF; k += 4) {
            __builtin_amdgcn_sched_barrier(0);
            typename M::Frag y[4][2];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    y[q][h] = alone(reinterpret_cast<const typename M::Frag*>(tile + (k + q) * 16 * kC + M::direct_at(l, 2 * p + h)));
            }
#pragma unroll
            for (int n = NS - 1; n >= 0; --n)
#pragma unroll
                for (int q = 0; q < 4; ++q) S.s[k + q] = M::mma(y[q][0], y[q][1], w[2 * p][n], w[2 * p + 1][n], S.s[k + q]);
        }
}

// acc[i] (token tile i) += a tile's columns times the state's rows 16 k .. + 31, split into terms.
template <typename T, int NS>
__device__ __forceinline__ void against_tokens(int l, const T* tile, int k, const typename Mat<T>::Frag (&s0)[NS],
                                               const typename Mat<T>::Frag (&s1)[NS], f32x4 (&acc)[4]) {
    using M = Mat<T>;
    typename M::Frag f[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[i][0] = M::transposed(l, tile + k * 16 * kC, i);
        f[i][1] = M::transposed(l, tile + (k + 1) * 16 * kC, i);
    }
#pragma unroll
    for (int n = NS - 1; n >= 0; --n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = M::mma(f[i][0], f[i][1], s0[n], s1[n], acc[i]);
}

__device__ __forceinline__ bool any_nonfinite(const f32x4 (&v)[4]) {
    float z = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) z = fmaf(v[i][r], 0.0f, z);
    return __ballot(!(z == 0.0f)) != 0;
}

// the multiplier of the state at one token
__device__ __forceinline__ float token_decay(const DeltaArgs& a, int64_t b, int64_t h, int64_t t, bool& cut) {
    float g = 0.0f;
    int pos = 1;
    if (t < a.seqlen) {
        pos = a.pos[b * a.seqlen + t];
        if (a.decay_mode == 2) g = a.decay[(b * a.heads + h) * a.seqlen + t];
        else if (a.decay_mode == 1) g = a.decay[h];
    }
    cut = pos == 0 || g <= kDecayCut;
    return cut ? 0.0f : expf(g);
}

__device__ __forceinline__ float lanes16(float v) {      // the sum over the 16 lanes of a row, in all of them
    v += __shfl_xor(v, 1);
    v += __shfl_xor(v, 2);
    v += __shfl_xor(v, 4);
    v += __shfl_xor(v, 8);
    return v;
}

// --------------------------------------------------------------------------------------------
// forward in time.  MODE kDeltaOut: the outs; kDeltaSum: a segment's end state from zeros, in further blocks from the
// identity's columns; kDeltaStates: what the backward needs.
// --------------------------------------------------------------------------------------------
template <typename T, typename TO, int KC, int VP, int MODE, int NS>
__global__ __launch_bounds__(VP * 4, 2) void delta_fwd_kernel(DeltaArgs a) {
    using M = Mat<T>;
    using Frag = typename M::Frag;
    constexpr int KF = KC / 16, kWaves = VP / 16, kThreads = VP * 4;
    constexpr bool kQ = MODE != kDeltaSum;
    using Smem = DeltaSmem<T, KC, VP, NS, kQ ? NS : 0, kQ, MODE == kDeltaStates ? 1 : 0>;
    constexpr bool kTwo = Smem::kBuffers == 2;
    __shared__ Smem smem;
    const int l = lane_id(), w = wave_id(), col = l & 15, g4 = (l >> 4) * 4, tid = threadIdx.x;
    const int64_t L = a.seqlen;
    const int mblocks = MODE == kDeltaSum ? (KC + VP - 1) / VP : 0, nseg = MODE == kDeltaSum ? a.sum_segs : a.nseg;
    const uint32_t id = walk_block((uint32_t)a.batch * a.heads * nseg * (1 + mblocks));
    const uint32_t rs = id / (uint32_t)(1 + mblocks), mb = id - rs * (1 + mblocks);     // mb: 0 the columns of v, else of the identity
    const uint32_t row = rs / (uint32_t)nseg, bat = row / (uint32_t)a.heads;
    const int64_t bh = row, b = bat, h = row - bat * a.heads, seg = rs - row * nseg;
    const int first = (int)seg * a.seg_chunks, last = min(a.chunks, first + a.seg_chunks) - 1;
    const T* kp = static_cast<const T*>(a.k) + (b * a.groups + h / (a.heads / a.groups)) * a.dk * L;
    const T* qp = static_cast<const T*>(a.q) + (b * a.groups + h / (a.heads / a.groups)) * a.dk * L;
    const int zf = w * 16, z = zf + col;
    const bool live = mb == 0 && z < a.dv;
    const uint32_t mask = live ? ~0u : 0u;
    const int64_t zrow = bh * a.dv + min(z, a.dv - 1);
    const T* vp = static_cast<const T*>(a.v) + zrow * L;
    const T* dop = MODE == kDeltaStates ? static_cast<const T*>(a.dout) + zrow * L : nullptr;
    TO* op = MODE == kDeltaOut ? static_cast<TO*>(a.out) + zrow * L : nullptr;
    T* ep = MODE == kDeltaStates ? static_cast<T*>(a.e) + zrow * L : nullptr;
    uint16_t* elp = MODE == kDeltaStates && M::kSplit ? a.e_low + zrow * L : nullptr;
    const float* betap = a.beta + bh * L;
    // half of the state's rows are none (1 x 2 heads of 24 x 32 x 256 tokens in fp32: a backward of 91.5 us, and 108 with all rows)
    const bool few = KF == 4 && a.dk <= 32;

    DeltaState<KF> S;
    const int64_t sz = (int64_t)a.dk * a.dv;
    if (MODE == kDeltaSum && mb == 0) S.load(nullptr, 0, 0, 0, 0);
    else if (MODE == kDeltaSum) S.identity((int)(mb - 1) * VP + zf, a.dk);
    else S.load(a.nseg > 1 ? a.seg + (bh * a.nseg + seg) * sz : a.entry ? a.entry + bh * sz : nullptr, a.dk, a.dv, zf, a.dv);

    FeatureRegs<T, KC, kThreads> kr, qr;
    ProductRegs<T, NS, kQ ? NS : 0, kThreads> hr;
    TokenRegs<T> vr, dr;
    f32x4 cr;
    // K, Q and the weights; H and P, which are needed later: half the loads at a time, each after products that
    // the memory's queues can drain under
    const auto load = [&](int chunk) {
        const int tid = here(threadIdx.x);
        kr.load(tid, kp, a.dk, chunk * kC, (int)L);
        if constexpr (kQ) qr.load(tid, qp, a.dk, chunk * kC, (int)L);
        const float* cf = a.coef + (bh * a.chunks + chunk) * kDeltaCoef;
        cr = *reinterpret_cast<const f32x4*>(cf + (tid < 48 ? tid * 4 : kCoefA));
    };
    const auto load_products = [&](int chunk) {
        const int tid = here(threadIdx.x);
        const int64_t unit = bh * a.chunks + chunk;
        hr.load(tid, a.products, unit);
    };
    const auto stage = [&](int chunk) {
        const int tid = here(threadIdx.x);
        auto& sm = smem.b[kTwo ? (chunk - first) & 1 : 0];
        const int64_t ct = (int64_t)chunk * kC;
        kr.settle(tid, kp, a.dk, ct, L);
        kr.store(tid, sm.k);
        if constexpr (kQ) {
            qr.settle(tid, qp, a.dk, ct, L);
            qr.store(tid, sm.q);
        }
        if (tid <= 48) *reinterpret_cast<f32x4*>(tid < 48 ? &sm.coef[0][0] + tid * 4 : sm.misc) = cr;
    };
    const auto stage_products = [&](int chunk) {
        const int tid = here(threadIdx.x);
        auto& sm = smem.b[kTwo ? (chunk - first) & 1 : 0];
        hr.store(tid, &sm.h[0][0][0], &sm.p[0][0][0]);
    };
    const auto flush = [&](int chunk) {
        if constexpr (MODE == kDeltaStates) {
            const auto& dot = smem.dot[(chunk - first) & 1][0];
            const int64_t t = (int64_t)chunk * kC + tid;
            if (tid < kC && t < L) {
                float v = dot[0][tid];
#pragma unroll
                for (int n = 1; n < kWaves; ++n) v += dot[n][tid];
                a.rq[bh * L + t] = v;
            }
        }
    };
    // The outs of a chunk are stored in the next, after its operands are in LDS: to wait for those, loaded a chunk ago, is to wait
    // for every store since.
    TokenRegs<TO> pending;
    bool any_pending = false;
    const auto store_pending = [&](int chunk) {
        if (MODE == kDeltaOut && any_pending && live) pending.store(op, (int64_t)chunk * kC, here(l), L);
    };
    bool all_cut = false;
    load(first);
    load_products(first);
    if constexpr (kTwo) {
        stage(first);
        stage_products(first);
        load(min(first + 1, last));
        load_products(min(first + 1, last));
    }
    for (int chunk = first; chunk <= last; ++chunk) {
        const int64_t ct = (int64_t)chunk * kC, unit = bh * a.chunks + chunk;
        auto& sm = smem.b[kTwo ? (chunk - first) & 1 : 0];
        auto& dot = smem.dot[(chunk - first) & 1][0];
        __syncthreads();
        if (MODE == kDeltaStates && chunk > first) flush(chunk - 1);
        if constexpr (kTwo) {
            stage(chunk + 1);
        } else {
            stage(chunk);
            stage_products(chunk);
            __syncthreads();
        }
        store_pending(chunk - 1);
        vr.load(vp, ct, here(l), L);                          // needed once K^T S is there
        if constexpr (MODE == kDeltaStates) dr.load(dop, ct, here(l), L);
        const float A = uniform(sm.misc[0]);
        const bool cut = A < 0.0f;
        all_cut = all_cut || cut;
        if (MODE == kDeltaSum && cut && mb > 0) {        // nothing that enters the segment leaves it
            S.clear();
            break;
        }
        const bool bad = __builtin_amdgcn_readfirstlane(__float_as_int(sm.misc[1])) != 0;
        if constexpr (MODE == kDeltaStates) {
            S.keep(a.states + (bh * delta_slots<T>(a.chunks) + chunk) * KC * VP, zf);
            if (!M::kSplit && chunk > 0 && chunk % a.bound_chunks == 0) {
                float* p = a.bound + ((bh * a.nb + chunk / a.bound_chunks - 1) * KF * kThreads + tid) * 4;
#pragma unroll
                for (int k = 0; k < KF; ++k) *reinterpret_cast<f32x4*>(p + k * 4 * kThreads) = S.s[k];
            }
        }
        // K^T S and Q^T S
        const int lk = here(l);                          // offsets computed anew in each phase: registers are short
        f32x4 ak[4], aq[4], x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) ak[i] = aq[i] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KF; k += 2) {
            if (k >= 2 && few) break;
            __builtin_amdgcn_sched_barrier(0);
            Frag s0[NS], s1[NS];
            M::template split<NS>(S.s[k], s0);
            M::template split<NS>(S.s[k + 1], s1);
            against_tokens<T, NS>(lk, sm.k, k, s0, s1, ak);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (kQ) against_tokens<T, NS>(lk, sm.q, k, s0, s1, aq);
        }
        load(min(chunk + 1 + kTwo, last));              // without a branch: the last chunks load theirs again
        if (kTwo) stage_products(chunk + 1);
        const int g4c = (here(l) >> 4) * 4;
        const auto four = [&](int which, int i) { return *reinterpret_cast<const f32x4*>(&sm.coef[which][i * 16 + g4c]); };
        Frag y[4][NS], vf[4];
        vr.get(mask, vf);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = M::widen(vf[i]) - ak[i] * four(0, i);
            M::template split<NS>(x[i] * four(2, i), y[i]);
        }
        f32x4 hx[4], u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) hx[i] = f32x4{0, 0, 0, 0};
        multiply_product<T, false, NS, NS>(l, sm.h, y, hx);
        load_products(min(chunk + 1 + kTwo, last));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] -= hx[i];                               // the errors
            u[i] = x[i] * four(2, i);
        }
        if (!bad && !any_nonfinite(u)) {
            if constexpr (kQ) {
                if constexpr (MODE == kDeltaStates) {
                    ErrorRegs<T> er;
                    er.set(x);
                    if (live) er.store(ep, elp, ct, here(l), L);
                }
                Frag uf[4][NS];
                f32x4 o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    M::template split<NS>(u[i], uf[i]);
                    o[i] = aq[i] * (four(0, i) * a.scale);
                }
                multiply_product<T, false, NS, NS>(l, sm.p, uf, o);
                if constexpr (MODE == kDeltaOut) {
                    any_pending = true;
                    pending.set(o);
                } else {
                    Frag df[4];
                    dr.get(mask, df);
#pragma unroll
                    for (int i = 0; i < 4; ++i) store_sum16(l, &dot[w][i * 16 + g4], sum16(o[i] * M::widen(df[i])));
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) M::template split<NS>(u[i] * four(1, i), y[i]);
            S.decay(cut ? 0.0f : A);                     // finite here
            add_tokens<T, KF, NS>(l, S, sm.k, y, few);
        } else {
            any_pending = false;
#pragma unroll 1
            for (int j = 0; j < kC; ++j) {
                const int64_t t = ct + j;
                bool start;
                const float mult = token_decay(a, b, h, t, start);
                if (start) S.clear();
                else S.decay(mult);
                const float beta = t < L ? betap[t] : 0.0f;
                const float e = (live && t < L ? Storage<T>::load1(vp + t) : 0.0f) - S.against(sm.k, j, mb > 0);
                const float ut = t < L ? beta * e : 0.0f;
                S.add(sm.k, j, ut);
                if constexpr (kQ) {
                    const float o = S.against(sm.q, j) * a.scale;
                    const bool mine = g4 == 0 && live && t < L;
                    if constexpr (MODE == kDeltaOut) {
                        if (mine) Storage<TO>::store1(op + t, o);
                    } else {
                        const float d = lanes16(live && t < L ? o * Storage<T>::load1(dop + t) : 0.0f);
                        if (l == 0) dot[w][j] = d;
                        if (mine) ErrorRegs<T>::put(ep + t, M::kSplit ? elp + t : nullptr, e);
                    }
                }
            }
        }
    }
    store_pending(last);
    if constexpr (MODE == kDeltaStates) {
        __syncthreads();
        flush(last);
        if (M::kSplit && last == a.chunks - 1 && a.bound_end) S.keep(a.states + (bh * delta_slots<T>(a.chunks) + a.chunks) * KC * VP, zf);
        if (!M::kSplit && last == a.chunks - 1 && a.bound_end) {
            float* p = a.bound + ((bh * a.nb + a.nb - 1) * KF * kThreads + tid) * 4;
#pragma unroll
            for (int k = 0; k < KF; ++k) *reinterpret_cast<f32x4*>(p + k * 4 * kThreads) = S.s[k];
        }
    }
    if constexpr (MODE == kDeltaSum) {
        if (mb == 0) {
            S.store(a.seg + (bh * a.nseg + seg) * sz, a.dk, a.dv, zf, a.dv);
            if (tid == 0) a.seg_cut[bh * a.nseg + seg] = all_cut;
        } else {
            S.store(a.seg_m + (bh * a.nseg + seg) * KC * KC, KC, KC, (int)(mb - 1) * VP + zf, KC);
        }
    } else if (MODE == kDeltaOut && a.leave && last == a.chunks - 1) {
        S.store(a.leave + bh * sz, a.dk, a.dv, zf, a.dv);
    }
}

// --------------------------------------------------------------------------------------------
// backwards in time: dv, the gradients that the states after the chunks get, and dbeta's and ddecay's parts; SUM: only
// the gradient that a segment adds
// --------------------------------------------------------------------------------------------
template <typename T, typename TO, int KC, int VP, bool SUM, int NS>
__global__ __launch_bounds__(VP * 4, 2) void delta_rev_kernel(DeltaArgs a) {
    using M = Mat<T>;
    using Frag = typename M::Frag;
    constexpr int KF = KC / 16, kWaves = VP / 16, kThreads = VP * 4;
    using Smem = DeltaSmem<T, KC, VP, NS, NS, true, SUM ? 0 : 2>;
    static_assert(Smem::kBuffers == 1, "one set of operands");
    __shared__ Smem smem;
    const int l = lane_id(), w = wave_id(), col = l & 15, g4 = (l >> 4) * 4, tid = threadIdx.x;
    const int64_t L = a.seqlen;
    const int nseg = SUM ? a.nseg - 1 : a.nseg;             // the first segment adds to nothing
    const uint32_t id = walk_block((uint32_t)a.batch * a.heads * nseg);
    const uint32_t row = id / (uint32_t)nseg, bat = row / (uint32_t)a.heads;
    const int64_t bh = row, b = bat, h = row - bat * a.heads, seg = id - row * nseg + (SUM ? 1 : 0);
    const int first = (int)seg * a.seg_chunks, last = min(a.chunks, first + a.seg_chunks) - 1;
    const T* kp = static_cast<const T*>(a.k) + (b * a.groups + h / (a.heads / a.groups)) * a.dk * L;
    const T* qp = static_cast<const T*>(a.q) + (b * a.groups + h / (a.heads / a.groups)) * a.dk * L;
    const int zf = w * 16, z = zf + col;
    const bool live = z < a.dv;
    const uint32_t mask = live ? ~0u : 0u;
    const int64_t zrow = bh * a.dv + min(z, a.dv - 1);
    const T* vp = static_cast<const T*>(a.v) + zrow * L;
    const T* dop = static_cast<const T*>(a.dout) + zrow * L;
    TO* op = SUM ? nullptr : static_cast<TO*>(a.out) + zrow * L;
    const T* ep = SUM ? nullptr : static_cast<const T*>(a.e) + zrow * L;
    const uint16_t* elp = !SUM && M::kSplit ? a.e_low + zrow * L : nullptr;
    T* wp = SUM || !a.w ? nullptr : static_cast<T*>(a.w) + zrow * L;      // a copy in T, where the out has another type
    uint16_t* wlp = !SUM && M::kSplit ? a.w_low + zrow * L : nullptr;
    const float* betap = a.beta + bh * L;
    const bool few = KF == 4 && a.dk <= 32;              // half of the state's rows are none

    DeltaState<KF> D;
    const int64_t sz = (int64_t)a.dk * a.dv;
    D.load(SUM ? nullptr : a.nseg > 1 ? a.seg + (bh * a.nseg + seg) * sz : a.entry ? a.entry + bh * sz : nullptr, a.dk, a.dv, zf, a.dv);

    FeatureRegs<T, KC, kThreads> kr, qr;
    ProductRegs<T, NS, NS, kThreads> hr;
    TokenRegs<T> vr, dr;
    ErrorRegs<T> er;
    f32x4 cr;
    const auto load = [&](int chunk) {
        const int tid = here(threadIdx.x);
        kr.load(tid, kp, a.dk, chunk * kC, (int)L);
        qr.load(tid, qp, a.dk, chunk * kC, (int)L);
        const float* cf = a.coef + (bh * a.chunks + chunk) * kDeltaCoef;
        cr = *reinterpret_cast<const f32x4*>(cf + (tid < 48 ? tid * 4 : kCoefA));
    };
    const auto load_products = [&](int chunk) {
        const int tid = here(threadIdx.x);
        const int64_t unit = bh * a.chunks + chunk;
        hr.load(tid, a.products, unit);
    };
    const auto stage = [&](int chunk) {
        const int tid = here(threadIdx.x);
        auto& sm = smem.b[0];
        const int64_t ct = (int64_t)chunk * kC;
        kr.settle(tid, kp, a.dk, ct, L);
        kr.store(tid, sm.k);
        qr.settle(tid, qp, a.dk, ct, L);
        qr.store(tid, sm.q);
        if (tid <= 48) *reinterpret_cast<f32x4*>(tid < 48 ? &sm.coef[0][0] + tid * 4 : sm.misc) = cr;
    };
    const auto stage_products = [&] {
        const int tid = here(threadIdx.x);
        auto& sm = smem.b[0];
        hr.store(tid, &sm.h[0][0][0], &sm.p[0][0][0]);
    };
    const auto bounded = [&](int chunk) { return chunk + 1 < a.chunks ? (chunk + 1) % a.bound_chunks == 0 : a.bound_end != 0; };
    const auto bound_of = [&](int next) { return (next + a.bound_chunks - 1) / a.bound_chunks; };
    const auto flush = [&](int chunk) {
        if constexpr (!SUM) {
            const auto& dot = smem.dot[(last - chunk) & 1];
            const int64_t t = (int64_t)chunk * kC + tid;
            if (tid < kC && t < L) {
                float v = dot[0][0][tid], d = dot[1][0][tid];
#pragma unroll
                for (int n = 1; n < kWaves; ++n) {
                    v += dot[0][n][tid];
                    d += dot[1][n][tid];
                }
                a.rk[bh * L + t] = -v;
                a.dbeta[bh * L + t] = d;
            }
            if (tid == kC && bounded(chunk)) {
                const float* x = smem.xdot[(last - chunk) & 1];
                float v = x[0];
#pragma unroll
                for (int n = 1; n < kWaves; ++n) v += x[n];
                a.dot[bh * (a.nb + 1) + bound_of(chunk + 1)] = v;
            }
        }
    };
    load(last);
    load_products(last);
    for (int chunk = last; chunk >= first; --chunk) {
        const int64_t ct = (int64_t)chunk * kC, unit = bh * a.chunks + chunk;
        auto& sm = smem.b[0];
        auto& dot = smem.dot[(last - chunk) & 1];
        __syncthreads();
        if (!SUM && chunk < last) flush(chunk + 1);
        stage(chunk);
        stage_products();
        dr.load(dop, ct, here(l), L);
        if constexpr (!SUM) {
            // a boundary at the chunk's end: the product of the state and its gradient there
            if (bounded(chunk)) {                            // block-uniform
                const int next = chunk + 1;
                float v = 0.0f;
                if constexpr (M::kSplit) {
                    v = D.dot_kept(a.states + (bh * delta_slots<T>(a.chunks) + next) * KC * VP, zf);
                } else {
                    const float* p = a.bound + ((bh * a.nb + bound_of(next) - 1) * KF * kThreads + tid) * 4;
#pragma unroll
                    for (int k = 0; k < KF; ++k) {
                        const f32x4 o = *reinterpret_cast<const f32x4*>(p + k * 4 * kThreads);
#pragma unroll
                        for (int r = 0; r < 4; ++r) v = fmaf(o[r], D.s[k][r], v);
                    }
                }
#pragma unroll
                for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
                if (l == 0) smem.xdot[(last - chunk) & 1][w] = v;
            }
            D.keep(a.grads + unit * KC * VP, zf);
        }
        __syncthreads();
        if constexpr (!SUM) {                            // needed late in the chunk
            vr.load(vp, ct, here(l), L);
            er.load(ep, elp, ct, here(l), L);
        }
        const float A = uniform(sm.misc[0]);
        const bool cut = A < 0.0f;
        const bool bad = __builtin_amdgcn_readfirstlane(__float_as_int(sm.misc[1])) != 0;
        const int lk = here(l);                          // offsets computed anew in each phase: registers are short
        f32x4 ak[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) ak[i] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KF; k += 2) {
            if (k >= 2 && few) break;
            __builtin_amdgcn_sched_barrier(0);
            Frag s0[NS], s1[NS];
            M::template split<NS>(D.s[k], s0);
            M::template split<NS>(D.s[k + 1], s1);
            against_tokens<T, NS>(lk, sm.k, k, s0, s1, ak);
        }
        load(max(chunk - 1, first));                    // without a branch: the last chunks load theirs again
        const int g4c = (here(l) >> 4) * 4;
        const auto four = [&](int which, int i) { return *reinterpret_cast<const f32x4*>(&sm.coef[which][i * 16 + g4c]); };
        f32x4 x[4];
        Frag df[4][1];                                   // exact: dout is of this type
        {
            Frag f[4];
            dr.get(mask, f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                df[i][0] = f[i];
                x[i] = ak[i] * four(1, i);
            }
            multiply_product<T, true, NS, 1>(l, sm.p, df, x);
        }
        Frag y[4][NS];
#pragma unroll
        for (int i = 0; i < 4; ++i) M::template split<NS>(x[i] * four(2, i), y[i]);
        f32x4 hx[4], dv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) hx[i] = f32x4{0, 0, 0, 0};
        multiply_product<T, true, NS, NS>(l, sm.h, y, hx);
        load_products(max(chunk - 1, first));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] -= hx[i];                               // du
            dv[i] = x[i] * four(2, i);
        }
        if (!bad && !any_nonfinite(x)) {
            if constexpr (!SUM) {
                TokenRegs<TO> out;
                out.set(dv);
                if (live) out.store(op, ct, here(l), L);
                if constexpr (sizeof(TO) != sizeof(T)) {
                    TokenRegs<T> copy;
                    copy.set(dv);
                    if (live) copy.store(wp, ct, here(l), L);
                }
                if constexpr (M::kSplit) {
                    HalfRegs low;
                    low.set_rest(dv);
                    if (live) low.store(wlp, ct, here(l), L);
                }
                Frag vf[4];
                vr.get(mask, vf);
#pragma unroll
                for (int i = 0; i < 4; ++i) store_sum16(l, &dot[0][w][i * 16 + g4], sum16(M::widen(vf[i]) * dv[i]));
                f32x4 e[4];
                er.get(mask, e);
#pragma unroll
                for (int i = 0; i < 4; ++i) store_sum16(l, &dot[1][w][i * 16 + g4], sum16(x[i] * e[i]));
            }
            D.decay(cut ? 0.0f : A);                     // finite here
#pragma unroll
            for (int i = 0; i < 4; ++i) M::template split<NS>(M::widen(df[i][0]) * (four(0, i) * a.scale), y[i]);
            add_tokens<T, KF, NS>(l, D, sm.q, y, few);
#pragma unroll
            for (int i = 0; i < 4; ++i) M::template split<NS>(-dv[i] * four(0, i), y[i]);
            add_tokens<T, KF, NS>(l, D, sm.k, y, few);
        } else {
#pragma unroll 1
            for (int j = kC - 1; j >= 0; --j) {
                const int64_t t = ct + j;
                const bool in = t < L;
                bool start;
                const float mult = token_decay(a, b, h, t, start);
                const float d = in && live ? Storage<T>::load1(dop + t) : 0.0f;
                D.add(sm.q, j, d * a.scale);
                const float du = D.against(sm.k, j), dvt = in ? betap[t] * du : 0.0f;
                if constexpr (!SUM) {
                    const float et = in && live ? ErrorRegs<T>::take(ep + t, M::kSplit ? elp + t : nullptr) : 0.0f;
                    const float vd = lanes16(in && live ? Storage<T>::load1(vp + t) * dvt : 0.0f), db = lanes16(in && live ? du * et : 0.0f);
                    if (l == 0) {
                        dot[0][w][j] = vd;
                        dot[1][w][j] = db;
                    }
                    if (g4 == 0 && live && in) {
                        Storage<TO>::store1(op + t, dvt);
                        if (wp) Storage<T>::store1(wp + t, dvt);
                        if constexpr (M::kSplit) wlp[t] = (uint16_t)rest_of(dvt, Mat<T>::round(f32x4{dvt, 0, 0, 0}).x << 16);
                    }
                }
                D.add(sm.k, j, -dvt);
                if (start) D.clear();
                else D.decay(mult);
            }
        }
    }
    if constexpr (!SUM) {
        __syncthreads();
        flush(first);
        if (a.leave && first == 0) D.store(a.leave + bh * sz, a.dk, a.dv, zf, a.dv);
    } else {
        D.store(a.seg + (bh * a.nseg + seg) * sz, a.dk, a.dv, zf, a.dv);
    }
}

// --------------------------------------------------------------------------------------------
// launches: one T, TO and KC in each translation unit
// --------------------------------------------------------------------------------------------
enum DeltaWalk : int {
    kWalkOut = 0, kWalkStates = 1, kWalkRev = 2, kWalkSum = 3, kWalkSumRev = 4
};

template <typename T, typename TO, int KC, int VP>
hipError_t launch_delta_vp(const DeltaArgs& a, DeltaWalk which, hipStream_t s) {
    constexpr int kAll = Mat<T>::kSplit ? 3 : 1;
    const int64_t rows = (int64_t)a.batch * a.heads, mblocks = (KC + VP - 1) / VP;
    const dim3 block(VP * 4), grid((unsigned)(rows * a.nseg));
    switch (which) {
        case kWalkOut: hipLaunchKernelGGL((delta_fwd_kernel<T, TO, KC, VP, kDeltaOut, kAll>), grid, block, 0, s, a); break;
        case kWalkStates: hipLaunchKernelGGL((delta_fwd_kernel<T, TO, KC, VP, kDeltaStates, kAll>), grid, block, 0, s, a); break;
        case kWalkRev: hipLaunchKernelGGL((delta_rev_kernel<T, TO, KC, VP, false, kAll>), grid, block, 0, s, a); break;
        case kWalkSum:
            hipLaunchKernelGGL((delta_fwd_kernel<T, TO, KC, VP, kDeltaSum, kAll>), dim3((unsigned)(rows * a.sum_segs * (1 + mblocks))),
                               block, 0, s, a);
            break;
        case kWalkSumRev:
            hipLaunchKernelGGL((delta_rev_kernel<T, TO, KC, VP, true, kAll>), dim3((unsigned)(rows * (a.nseg - 1))), block, 0, s, a);
            break;
    }
    return hipGetLastError();
}

template <typename T, typename TO, int KC>
hipError_t launch_delta_kc(const DeltaArgs& a, DeltaWalk which, hipStream_t s) {
    return a.dv <= 64 ? launch_delta_vp<T, TO, KC, 64>(a, which, s) : launch_delta_vp<T, TO, KC, 128>(a, which, s);
}

}  // namespace pm
