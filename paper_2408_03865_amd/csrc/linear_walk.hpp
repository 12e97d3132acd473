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
// Mapping.  One block walks a row (or a segment of it) of one head; activations are (features, tokens),
// tokens innermost.  A chunk's tiles sit in LDS as they do in memory.  Products
// over tokens (z and the update) read their operands directly, four tokens a lane; products over
// features (x . y and x . S) read them transposed (ds_read_b64_tr_b16 in bf16).  The waves share the
// 64 x 64 products of x and y by strips of 16 x's and pass them, weighted and rounded to T, through
// LDS.  Each wave owns 16 of z's features, and of x's all or half: its part of S stays in registers, in
// the layout that an MFMA result has and, four rows of it a lane, an MFMA operand takes.
// What bounds it: the waves' own work between three barriers a chunk, none of the units alone.  8 x 64 heads x
// 4096 tokens, dk 128 and dv 64, bf16, forward: 311 to 345 us on different cards; the VALU issues 57% of the cycles (weights, the splits of S and of
// weighted z), LDS is read and written in 53% (every wave reads all of x and y for its part of z), the matrix units are
// busy 19%; 682 MB move at 2.1 TB/s.  8 x 32 heads, 128 and 128, backward 1409 us; of it, in a trace whose kernels are 14%
// slower, dq 552 (VALU 68%, LDS 36%, matrix 22%), dk 540, dv 325.  In fp32 the matrix units bound them: forward 930 us, busy
// 65% (VALU 15%, LDS 18%), backward 3392.
// Longer chunks would do more products inside a chunk, shorter ones split S more often.
// Rounding in bf16: the weighted products x . y and, in plain walks, the copy of S that is
// multiplied with x are rounded to bf16 once (each enters the out alone, which a bf16 output rounds as
// much once more; a 32-bit output of bf16 inputs has their accuracy); what S itself adds is split into
// two or three bf16 terms that hold 16 or all 24 bits of it, and in the walks that feed the decay's
// gradient so is the copy of S.
//
// Infinities and NaN reach the outs whose sums hold them and no other: masks select, a chunk whose y or z
// holds one takes plain loops over the unmasked pairs in place of the matrix products over tokens, where 0
// times it would spread, and the decays are summed in the walk's direction (chunk_decay).
#pragma once

#include "common.hpp"
#include "linear.hpp"

namespace pm {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kC = (int)kLinChunk;

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// v, as a value that is new here: what is computed from it stays where it is used, and takes no
// registers elsewhere.
__device__ __forceinline__ int here(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// The same where HIDE, for offsets that a kernel short of registers computes anew in each phase.
template <bool HIDE>
__device__ __forceinline__ int fresh(int v) {
    if constexpr (HIDE) return here(v);
    else return v;
}

// A decay below this multiplies by 0 in 32 bits (exp(-104) < 2^-150): the token is taken for a start.
constexpr float kDecayCut = -104.0f;

// --------------------------------------------------------------------------------------------
// matrix operands: four values of the contracted index a lane, 4 (lane / 16) .. + 3 of 16, for
// row or column lane % 16 -- also the layout of a 16 x 16 result, contracted along its rows.
// Tiles in LDS are rows of 64 tokens without padding; the 16-byte pieces of row r are permuted by
// an exclusive or with swz(r), so that 16 rows by 16 tokens, read either way, take every bank once.
// --------------------------------------------------------------------------------------------
template <typename T> struct Mat;

template <> struct Mat<bf16_t> {
    typedef u32x2 Frag;
    static constexpr bool kSplit = true;
    __device__ static int swz(int r) { return (r & 6) | ((r >> 3) & 1); }
    // rows 0..15 of the tile, tokens 16 tt + 4 (lane / 16) .. + 3 of row lane % 16
    __device__ static int direct_at(int l, int tt) {
        const int r = l & 15, half = (l >> 5) ^ ((r >> 3) & 1);
        return r * kC + half * 8 + ((l >> 4) & 1) * 4 + (tt ^ ((r >> 1) & 3)) * 16;
    }
    __device__ static Frag direct(int l, const bf16_t* p, int tt) { return *reinterpret_cast<const u32x2*>(p + direct_at(l, tt)); }
    // rows 4 (lane / 16) .. + 3 of the tile, token 16 tt + lane % 16
    __device__ static Frag transposed(int l, const bf16_t* p, int tt) {
        const int r = (l >> 4) * 4 + ((l & 15) >> 2), half = ((l >> 1) & 1) ^ ((r >> 3) & 1);
        const bf16_t* q = p + r * kC + half * 8 + (l & 1) * 4 + (tt ^ ((r >> 1) & 3)) * 16;
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
    // 0 times every value, added up: NaN if one is infinite or NaN
    __device__ static float zero_sum(const u32x4& w, float v) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, uint32_t(w[i])), bf16x2{0, 0}, v, false);
        return v;
    }
};

template <> struct Mat<float> {
    typedef f32x4 Frag;
    static constexpr bool kSplit = false;
    __device__ static int swz(int r) { return r & 15; }
    __device__ static int direct_at(int l, int tt) {
        const int r = l & 15;
        return r * kC + ((l >> 4) ^ (r & 3)) * 4 + (tt ^ (r >> 2)) * 16;
    }
    __device__ static Frag direct(int l, const float* p, int tt) { return *reinterpret_cast<const f32x4*>(p + direct_at(l, tt)); }
    __device__ static Frag transposed(int l, const float* p, int tt) {
        const int g = l >> 4;
        const float* q = p + g * 4 * kC + (tt ^ g) * 16 + (l & 3);
        Frag v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = q[e * kC + (((l >> 2) & 3) ^ e) * 4];
        return v;
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
    __device__ static float zero_sum(const u32x4& w, float v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v = fmaf(__uint_as_float(w[i]), 0.0f, v);
        return v;
    }
};

// The value of row r at token t of a tile.
template <typename T>
__device__ __forceinline__ float tile_value(const T* tile, int r, int t) {
    constexpr int kPer = Storage<T>::kPerVec;
    return Storage<T>::load1(tile + r * kC + ((t / kPer) ^ Mat<T>::swz(r)) * kPer + t % kPer);
}

// --------------------------------------------------------------------------------------------
// a chunk's decays
// --------------------------------------------------------------------------------------------
struct __attribute__((aligned(16))) ChunkDecay {
    float hi[kC], lo[kC];       // G in log2 units, as a sum of two floats
    float in[kC], up[kC];       // scaled; 0 where the term is left out
    int32_t start[kC];          // the last start up to the token, -1: none in the chunk
    float a;                    // -1: a start in the chunk
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

// Whether token t takes the state that enters the chunk (enters), and whether it adds to the one that
// leaves it (leaves), in a forward walk; a reverse walk has the two the other way round.
template <bool REV>
__device__ __forceinline__ bool enters(const ChunkDecay& c, int t) {
    return REV ? t >= c.start[kC - 1] : c.start[t] < 0;
}
template <bool REV>
__device__ __forceinline__ bool leaves(const ChunkDecay& c, int t) {
    return enters<!REV>(c, t);
}
// Whether x's out takes y.
template <bool REV>
__device__ __forceinline__ bool takes(const ChunkDecay& c, int x, int y) {
    return REV ? x <= y && c.start[y] <= x : y <= x && c.start[x] <= y;
}

// One step of the segmented sum over lanes: a lane that has no start among those summed so far adds the sum of
// the lane that CTRL names, and takes its start.
template <int CTRL, int ROWS>
__device__ __forceinline__ void scan_step(double& v, int& start) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, CTRL, ROWS, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(bits >> 32), CTRL, ROWS, 0xf, false);
    const int ps = __builtin_amdgcn_update_dpp(-1, start, CTRL, ROWS, 0xf, false);
    if (start < 0) {
        v += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
        start = ps;
    }
}

__device__ __forceinline__ void scan_lanes(double& v, int& start) {
    scan_step<row_shr(1), 0xf>(v, start);
    scan_step<row_shr(2), 0xf>(v, start);
    scan_step<row_shr(4), 0xf>(v, start);
    scan_step<row_shr(8), 0xf>(v, start);
    scan_step<0x142, 0xa>(v, start);     // lane 15 of rows 0 and 2 to the rows after them
    scan_step<0x143, 0xc>(v, start);     // lane 31 to rows 2 and 3
}

// The chunk's token whose decay a lane loads: the sums run over the lanes.
template <bool REV>
__device__ __forceinline__ int decay_token(int l) {
    return REV ? kC - 1 - here(l) : l;      // computed anew: kept over the loop it is a register too many
}

// The value of one lane, in all.
__device__ __forceinline__ double uniform(double v, int lane) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(bits >> 32), lane) << 32 |
                                          (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)bits, lane));
}

// The value of the lane before, 0 in lane 0.
__device__ __forceinline__ int lane_before(int v) { return __builtin_amdgcn_update_dpp(0, v, 0x138, 0xf, 0xf, false); }

// One wave, lane l = token decay_token(l).  The sum is kept in 64 bits and starts anew at each start, so that no
// sequence's decays reach another's.  In a reverse walk G is minus the sum of the decays after the token, up to the
// chunk's or the sequence's end (differences of G are the same): whichever way the walk goes, a sum that holds an
// infinite decay or a NaN belongs to a token whose out holds it too, by a pair or by the state, and pairs on its
// other side do not meet it.
template <bool REV>
__device__ __forceinline__ void chunk_decay(const TokenDecay& d, ChunkDecay& c, float iscale, float uscale) {
    const int l = lane_id(), tok = decay_token<REV>(l);
    const bool cut = d.pos == 0 || d.g <= kDecayCut;
    double v = cut ? 0.0 : (double)d.g * 1.4426950408889634;
    if constexpr (!REV) {
        int start = cut ? l : -1;
        scan_lanes(v, start);
        const float hi = (float)v, lo = (float)(v - (double)hi);
        const float ehi = __shfl(hi, 63), elo = __shfl(lo, 63);
        const int estart = __shfl(start, 63);
        const float first = start < 0 ? fast_exp2(hi + lo) : 0.0f;
        const float last = l >= estart ? pair_decay(ehi, elo, hi, lo) : 0.0f;
        c.hi[tok] = hi;
        c.lo[tok] = lo;
        c.start[tok] = start;
        c.in[tok] = first * iscale;
        c.up[tok] = last * uscale;
        if (l == 63) c.a = start < 0 ? first : -1.0f;
    } else {
        const uint64_t starts = __builtin_bitreverse64(__ballot(cut));      // bit: token
        const uint64_t bits = __builtin_bit_cast(uint64_t, v);
        const double own = uniform(v, 63);
        v = __builtin_bit_cast(double, (uint64_t)(uint32_t)lane_before((int)(uint32_t)(bits >> 32)) << 32 |
                                           (uint32_t)lane_before((int)(uint32_t)bits));
        int after = lane_before(cut ? 1 : 0) - 1;       // 0: a start among the tokens after it, -1: none
        scan_lanes(v, after);
        const float hi = (float)v, lo = (float)(v - (double)hi);
        const double all = own + uniform(v, 63);        // of the tokens before the first start
        const uint64_t upto = starts << here(l);        // bit 63: the token
        const float first = upto == 0 ? fast_exp2((float)(all - v)) : 0.0f;
        c.hi[tok] = -hi;
        c.lo[tok] = -lo;
        c.start[tok] = upto ? tok - __builtin_clzll(upto) : -1;
        c.in[tok] = after < 0 ? fast_exp2(hi + lo) * iscale : 0.0f;
        c.up[tok] = first * uscale;
        if (l == 0) c.a = starts ? -1.0f : first;
    }
}

// --------------------------------------------------------------------------------------------
// tiles: ROWS features x 64 tokens through registers into LDS; features and tokens that the tensor
// lacks are 0
// --------------------------------------------------------------------------------------------
__device__ const u32x4 walk_zero = {0, 0, 0, 0};

template <typename T, int ROWS, int THREADS>
struct TileRegs {
    static constexpr int kPer = Storage<T>::kPerVec, kLanes = kC / kPer, kRowsPass = THREADS / kLanes;
    static constexpr int kPasses = ROWS / kRowsPass;
    static_assert(kRowsPass % 16 == 0 && ROWS % kRowsPass == 0, "a thread's rows are permuted alike");
    u32x4 w[kPasses];

    // Every lane loads whole vectors from inside its row, a row that the tensor has, whatever it needs: a branch
    // here would make the kernel wait for the loads at once.  settle() puts right what the last chunk of a row
    // and heads of fewer features need, when the values are used.  at: offset_of(), the same for all tensors.
    __device__ static uint32_t offset_of(int tid, int t0, int L) {
        const int tok = (tid % kLanes) * kPer;
        return L < kPer ? 0u : ((uint32_t)(tid / kLanes) * (uint32_t)L + (uint32_t)min(t0 + tok, L - kPer)) * (uint32_t)sizeof(T);
    }
    __device__ void load(int tid, uint32_t at, const T* p, int rows, int L) {
        // said to be global memory, which the compiler cannot see of a choice of two pointers: what it then
        // loads makes every wait for LDS wait for memory too
        typedef const __attribute__((address_space(1))) char* Bytes;
        typedef const __attribute__((address_space(1))) typename Storage<T>::Vec* Global;
        const int row0 = tid / kLanes;
        Bytes base = (Bytes)(uintptr_t)(L < kPer ? reinterpret_cast<const T*>(&walk_zero) : p);
        const int64_t apart = L < kPer ? 0 : (int64_t)kRowsPass * L * (int64_t)sizeof(T);
        if (rows == ROWS) {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) w[i] = *(Global)(base + i * apart + at);
        } else {
            const uint32_t first = L < kPer ? 0u : at - (uint32_t)row0 * (uint32_t)L * (uint32_t)sizeof(T);    // in the pass's first row
#pragma unroll
            for (int i = 0; i < kPasses; ++i)
                w[i] = *(Global)(base + (i * kRowsPass < rows ? i * apart : 0) + (row0 + i * kRowsPass < rows ? at : first));
        }
    }
    __device__ void settle(int tid, const T* p, int rows, int64_t t0, int64_t L) {
        const int row0 = tid / kLanes, tok = (tid % kLanes) * kPer;
        if (rows < ROWS) {
#pragma unroll
            for (int i = 0; i < kPasses; ++i)
                if (row0 + i * kRowsPass >= rows) w[i] = u32x4{0, 0, 0, 0};
        }
        if (t0 + kC <= L) return;
        if (L < kPer) {                     // rows shorter than a vector
#pragma unroll 1
            for (int i = 0; i < kPasses; ++i) {
                const int row = row0 + i * kRowsPass;
                u32x4 v = {0, 0, 0, 0};
#pragma unroll 1
                for (int k = 0; k < kPer; ++k) push(v, row < rows && tok + k < L ? p[row * L + tok + k] : T{});
#pragma unroll
                for (int j = 0; j < kPasses; ++j)
                    if (j == i) w[j] = v;
            }
            return;
        }
        const int64_t over = t0 + tok + kPer - L;           // elements that the vector was read too early
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            u32x4 v = over >= kPer ? u32x4{0, 0, 0, 0} : w[i];
#pragma unroll
            for (int k = 1; k < kPer; ++k) {
                u32x4 u = v;
                push(u, T{});
                v = over >= k && over < kPer ? u : v;
            }
            w[i] = v;
        }
    }
    // v after the last of the vector's elements, whose first leaves
    __device__ static void push(u32x4& w, bf16_t v) {
        w = u32x4{__builtin_amdgcn_alignbit(w.y, w.x, 16), __builtin_amdgcn_alignbit(w.z, w.y, 16),
                  __builtin_amdgcn_alignbit(w.w, w.z, 16), __builtin_amdgcn_alignbit(v.bits, w.w, 16)};
    }
    __device__ static void push(u32x4& w, float v) { w = u32x4{w.y, w.z, w.w, __float_as_uint(v)}; }
    __device__ void store(int tid, T* tile) const {
        const int row0 = tid / kLanes;
        T* p = tile + row0 * kC + ((tid % kLanes) ^ Mat<T>::swz(row0)) * kPer;
#pragma unroll
        for (int i = 0; i < kPasses; ++i) *reinterpret_cast<u32x4*>(p + i * kRowsPass * kC) = w[i];
    }
    __device__ float zero_sum(float v) const {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) v = Mat<T>::zero_sum(w[i], v);
        return v;
    }
};

template <typename T>
__device__ __forceinline__ const T* head_base(const WalkTensor& t, int64_t b, int64_t h, int heads, int64_t L) {
    return static_cast<const T*>(t.p) + ((b * t.heads + (uint32_t)h / (uint32_t)(heads / t.heads)) * t.rows) * L;
}

// The block's place: heads that share tensors run on one XCD, whose L2 then holds them (blocks go to
// the 8 XCDs in turn).
__device__ __forceinline__ uint32_t walk_block(uint32_t n) {
    const uint32_t id = blockIdx.x, per = n / 8;
    return id < per * 8 ? (id % 8) * per + id / 8 : id;
}

// The same for blocks of single chunks, `inner` blocks a chunk: eight chunks in a row to an XCD, whose pieces of 128 bytes make
// up 1 KB of a feature's row, and all blocks of a chunk.
__device__ __forceinline__ uint32_t chunk_block(uint32_t inner) {
    const uint32_t id = blockIdx.x, span = 64 * inner, r = id % span, first = id - r;
    return first + span <= gridDim.x ? first + (r % 8) * (8 * inner) + r / 8 : id;
}

// --------------------------------------------------------------------------------------------
// the state: 16 z features a wave, and of the x features all or half: KF tiles of 16 by 16
// --------------------------------------------------------------------------------------------
template <int KF>
struct State {
    f32x4 s[KF];
    int xf, zf;                         // the wave's first x and z feature

    template <typename F>
    __device__ void each(F f) {         // f(x feature of the lane's first value, z feature, its four values)
        const int l = here(lane_id());
#pragma unroll
        for (int k = 0; k < KF; ++k) f(xf + k * 16 + (l >> 4) * 4, zf + (l & 15), s[k]);
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
    __device__ void decay(bool cut, float a) {      // both the same for the whole wave
        if (cut) {
#pragma unroll
            for (int k = 0; k < KF; ++k) s[k] = f32x4{0, 0, 0, 0};
        } else {
#pragma unroll
            for (int k = 0; k < KF; ++k) s[k] *= a;
        }
    }
};

__device__ __forceinline__ float uniform(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
}

// S <- A S + sum_j up_j y_j z_j^T
template <typename T, bool REV, int NS, int KF>
__device__ __forceinline__ void update(State<KF>& S, const T* ys, const T* zs, const ChunkDecay& c, bool cut, bool bad) {
    using M = Mat<T>;
    const int l = here(lane_id()), four = (l >> 4) * 4;
    ys += S.xf * kC;
    zs += S.zf * kC;
    S.decay(cut, uniform(c.a));
    if (bad) {
        const int lb = here(l);
#pragma unroll 1
        for (int j = 0; j < kC; ++j) {
            if (!leaves<REV>(c, j)) continue;
            const float zv = tile_value(zs, lb & 15, j) * c.up[j];
#pragma unroll
            for (int k = 0; k < KF; ++k) {
#pragma unroll
                for (int r = 0; r < 4; ++r) S.s[k][r] = fmaf(tile_value(ys + k * 16 * kC, (lb >> 4) * 4 + r, j), zv, S.s[k][r]);
                __builtin_amdgcn_sched_barrier(0);      // few values at a time: registers count, not speed
            }
        }
        return;
    }
#pragma unroll
    for (int p = 0; p < 2; ++p) {                               // 32 tokens
        typename M::Frag zw[2][NS];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const f32x4 up = *reinterpret_cast<const f32x4*>(&c.up[(2 * p + q) * 16 + four]);
            M::template split<NS>(M::widen(M::direct(l, zs, 2 * p + q)) * up, zw[q]);
        }
#pragma unroll
        for (int k = 0; k < KF; ++k) {
            const typename M::Frag y0 = M::direct(l, ys + k * 16 * kC, 2 * p), y1 = M::direct(l, ys + k * 16 * kC, 2 * p + 1);
#pragma unroll
            for (int n = 0; n < NS; ++n) S.s[k] = M::mma(y0, y1, zw[0][n], zw[1][n], S.s[k]);
        }
    }
}

// The four values' sums over the 16 lanes of a row: lane 7 has those of x and z, lane 15 of y and w.
__device__ __forceinline__ f32x2 sum16(const f32x4& v) {
    return f32x2{row_sum2_to_7_15(v.x, v.y), row_sum2_to_7_15(v.z, v.w)};
}
// and their place: two floats of four consecutive ones, from lanes 7 and 15
__device__ __forceinline__ void store_sum16(int l, float* four, const f32x2& s) {
    if ((l & 7) == 7) {
        float* p = four + ((l >> 3) & 1);
        p[0] = s.x;
        p[2] = s.y;
    }
}

// Parts: in bf16 the x features can be split over two waves, so that twice the waves share a chunk's latencies; each
// multiplies x with its half of the state for all tokens, and the sums meet in LDS.  One part has fewer waves,
// but more blocks to a CU, and does less in all: plain walks of heads of up to 64 features take it from 768 blocks
// on.  Us with one part and two (batch x heads x 4096 tokens, forward): dk and dv 64, 4 x 64 231, 185; 8 x 64 281, 283;
// 12 x 64 338, 408; 16 x 64 413, 511; dk 128, dv 64, 8 x 64 402, 382; 16 x 64 718, 679; the whole backward of 8 x 32 heads,
// dk and dv 128, 2068, 1477.
template <typename T, int KC, int VP>
constexpr int walk_parts() {
    return sizeof(T) == 2 && KC >= VP ? 2 : 1;
}
template <typename T, int KC, int VP, int MODE, int kParts>
struct WalkSmem {
    static constexpr int kWaves = VP / 16 * kParts;
    __attribute__((aligned(16))) T x[KC * kC];
    __attribute__((aligned(16))) T y[KC * kC];
    __attribute__((aligned(16))) T z[VP * kC];
    __attribute__((aligned(16))) T e[MODE != kWalkPlain ? VP * kC : 8];
    __attribute__((aligned(16))) T p[kC * kC];          // x's rows
    __attribute__((aligned(16))) f32x4 half[kParts == 2 ? kWaves * 2 * 64 : 1];        // sums for the other part's tokens
    ChunkDecay c[2];
    __attribute__((aligned(16))) float rsum[MODE == kWalkDq ? kWaves / 4 : 1][kC];
    __attribute__((aligned(16))) float csum[MODE == kWalkDq ? 4 : 1][kC];
    __attribute__((aligned(16))) float dot[MODE != kWalkPlain ? VP / 16 : 1][kC];
    float xdot[kWaves];
};

// Waves of a SIMD that the registers are to leave room for.
template <typename T, int KC, int VP, int MODE>
constexpr int walk_waves() {
    if (sizeof(T) == 4) return VP == 64 ? 1 : 2;
    return 4;
}
constexpr int walk_threads(int VP, int parts) { return VP * 4 * parts; }

// Wave (z tile, part): 16 of z's features, and of the x features and the out's tokens all or, of two waves,
// half.  All waves share the products of x and y by strips of 16 x's and parts of the y's.
template <typename T, typename TO, int KC, int VP, int MODE, bool REV, int NS, int NO, int kParts>
__global__ __launch_bounds__((walk_threads(VP, kParts)), (walk_waves<T, KC, VP, MODE>())) void walk_kernel(WalkArgs a) {
    using M = Mat<T>;
    using Frag = typename M::Frag;
    constexpr int KT = KC / 16, VT = VP / 16, KF = KT / kParts, XT = 4 / kParts;
    constexpr int kWaves = VT * kParts, kThreads = kWaves * 64, kYParts = kWaves / 4, kYTiles = 4 / kYParts;
    // short of registers
    constexpr bool kTight = MODE != kWalkPlain || VP > KC || (REV && kParts < walk_parts<T, KC, VP>());
    __shared__ WalkSmem<T, KC, VP, MODE, kParts> sm;
    const int l = lane_id(), w = wave_id();
    const int64_t L = a.seqlen;
    const uint32_t id = walk_block((uint32_t)a.batch * a.heads * a.nseg);       // at most 2^23 of them
    const uint32_t row = id / (uint32_t)a.nseg, bat = row / (uint32_t)a.heads;
    const int64_t bh = row, b = bat, h = row - bat * a.heads, seg = id - row * a.nseg;
    const int chunks = (int)((L + kC - 1) / kC);
    const int first = (int)seg * a.seg_chunks, last = min(chunks, first + a.seg_chunks) - 1;
    const T* xp = head_base<T>(a.x, b, h, a.heads, L);
    const T* yp = head_base<T>(a.y, b, h, a.heads, L);
    const T* zp = head_base<T>(a.z, b, h, a.heads, L);
    const T* ep = MODE != kWalkPlain ? head_base<T>(a.e, b, h, a.heads, L) : nullptr;
    const int part = w / VT, ztile = w % VT;
    TO* op = static_cast<TO*>(a.out) + (bh * a.z.rows + ztile * 16) * L;        // the wave's first z feature

    State<KF> S;
    S.xf = part * KF * 16;
    S.zf = ztile * 16;
    const int64_t sz = (int64_t)a.x.rows * a.z.rows;
    S.load(a.nseg > 1 ? a.seg + (bh * a.nseg + seg) * sz : a.entry ? a.entry + bh * sz : nullptr, a);

    // boundary n of the row, 1 to nb: the state there, stored (dq) or multiplied with the one that dq stored (dk)
    const auto bound_at = [&](int64_t n) {
        return a.bound + ((bh * a.nb + n - 1) * KF * kThreads + here(threadIdx.x)) * 4;
    };
    const auto bound_store = [&](int64_t n) {
        float* p = bound_at(n);
#pragma unroll
        for (int k = 0; k < KF; ++k) *reinterpret_cast<f32x4*>(p + k * 4 * kThreads) = S.s[k];
    };
    const auto bound_dot = [&](int64_t n) {              // block-uniform
        const float* p = bound_at(n);
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < KF; ++k) {
            const f32x4 o = *reinterpret_cast<const f32x4*>(p + k * 4 * kThreads);
#pragma unroll
            for (int r = 0; r < 4; ++r) v = fmaf(o[r], S.s[k][r], v);
        }
#pragma unroll
        for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
        __syncthreads();
        if (l == 0) sm.xdot[w] = v;
        __syncthreads();
        if (threadIdx.x == 0) {
            v = sm.xdot[0];
#pragma unroll
            for (int i = 1; i < kWaves; ++i) v += sm.xdot[i];
            a.dot[bh * (a.nb + 1) + n] = v;
        }
    };

    TileRegs<T, KC, kThreads> xr, yr;
    TileRegs<T, VP, kThreads> zr, er;
    TokenDecay td{0.0f, 1};
    const int coef_wave = REV ? 3 : kYParts > 1 ? 4 : 0;    // a wave with the fewest products of x and y
    const auto load = [&](int chunk) {
        const int tid = fresh<kTight>(threadIdx.x);
        const uint32_t at = TileRegs<T, KC, kThreads>::offset_of(tid, chunk * kC, (int)L);
        xr.load(tid, at, xp, a.x.rows, (int)L);
        yr.load(tid, at, yp, a.y.rows, (int)L);
        zr.load(tid, at, zp, a.z.rows, (int)L);
        if constexpr (MODE != kWalkPlain) er.load(tid, at, ep, a.e.rows, (int)L);
    };
    const auto load_td = [&](int chunk) {
        if (w == coef_wave) td = load_decay(a, b, h, (int64_t)chunk * kC + decay_token<REV>(l));
    };
    // the decay's part of a finished chunk, from the waves' sums
    const auto flush_r = [&](int chunk) {
        if constexpr (MODE != kWalkPlain) {
            const int64_t t = (int64_t)chunk * kC + threadIdx.x;
            if (threadIdx.x < kC && t < L) {
                const int i = threadIdx.x;
                float v = sm.dot[0][i];
#pragma unroll
                for (int n = 1; n < VT; ++n) v += sm.dot[n][i];
                if constexpr (MODE == kWalkDq) {
#pragma unroll
                    for (int n = 0; n < kYParts; ++n) v += sm.rsum[n][i];
                    v -= (sm.csum[0][i] + sm.csum[1][i]) + (sm.csum[2][i] + sm.csum[3][i]);
                }
                a.r[bh * L + t] = v;
            }
        }
    };

    constexpr int step = REV ? -1 : 1;
    const int begin = REV ? last : first, n = last - first + 1;
    if (threadIdx.x == 0) sm.c[0].bad[0] = sm.c[1].bad[0] = 0;
    load_td(begin);
    load(begin);
    if (w == coef_wave) chunk_decay<REV>(td, sm.c[0], a.iscale, a.uscale);
    if (n > 1) load_td(begin + step);
    for (int it = 0; it < n; ++it) {
        const int chunk = begin + it * step, tid = fresh<kTight>(threadIdx.x);
        ChunkDecay& c = sm.c[it & 1];
        __syncthreads();                                // the tiles of the chunk before are read
        if (it > 0) flush_r(chunk - step);
        const int64_t ct = (int64_t)chunk * kC;
        xr.settle(tid, xp, a.x.rows, ct, L);
        yr.settle(tid, yp, a.y.rows, ct, L);
        zr.settle(tid, zp, a.z.rows, ct, L);
        if constexpr (MODE != kWalkPlain) er.settle(tid, ep, a.e.rows, ct, L);
        xr.store(tid, sm.x);
        yr.store(tid, sm.y);
        zr.store(tid, sm.z);
        if constexpr (MODE != kWalkPlain) er.store(tid, sm.e);
        if (zr.zero_sum(yr.zero_sum(0.0f)) != 0.0f) c.bad[0] = 1;
        if constexpr (MODE == kWalkDq) {
            if (chunk > 0 && chunk % a.bound_chunks == 0) bound_store(chunk / a.bound_chunks);
        }
        if constexpr (MODE == kWalkDk) {
            const int next = chunk + 1;
            if (next < chunks ? next % a.bound_chunks == 0 : a.bound_end != 0)
                bound_dot((next + a.bound_chunks - 1) / a.bound_chunks);
        }
        __syncthreads();
        if (it + 1 < n) load(chunk + step);     // the next chunk's tiles, during this one

        const bool cut = __builtin_amdgcn_readfirstlane(__float_as_int(c.a)) < 0;      // a sequence starts in the chunk
        // products of x and y, weighted: 16 x's by all y's, or a part of them
        {
            const int l = fresh<kTight>(lane_id()), col = l & 15, four = (l >> 4) * 4;
            if (w == coef_wave && it + 1 < n) {
                ChunkDecay& cn = sm.c[(it + 1) & 1];
                chunk_decay<REV>(td, cn, a.iscale, a.uscale);
                if (l == 0) cn.bad[0] = 0;
                if (it + 2 < n) load_td(chunk + 2 * step);
            }
            const int strip = w % 4, ypart = w / 4;
            Frag xf[KT];
#pragma unroll
            for (int k = 0; k < KT; ++k) xf[k] = M::transposed(l, sm.x + k * 16 * kC, strip);
            const int xt = strip * 16 + col;
            const float xhi = c.hi[xt], xlo = c.lo[xt];
            float rs = 0.0f;
#pragma unroll 1
            for (int i = 0; i < kYTiles; ++i) {
                const int yt = ypart * kYTiles + i;
                f32x4 d = {0, 0, 0, 0};
                Frag* pp = reinterpret_cast<Frag*>(sm.p + strip * 16 * kC + M::direct_at(l, yt));
                f32x4 cs = {0, 0, 0, 0};
                if (REV ? yt >= strip : yt <= strip) {
#pragma unroll
                    for (int k = 0; k < KT; k += 2)
                        d = M::mma(M::transposed(l, sm.y + k * 16 * kC, yt), M::transposed(l, sm.y + (k + 1) * 16 * kC, yt), xf[k],
                                   xf[k + 1], d);
                    const int y0 = yt * 16 + four;
                    const f32x4 yhi = *reinterpret_cast<const f32x4*>(&c.hi[y0]), ylo = *reinterpret_cast<const f32x4*>(&c.lo[y0]);
                    f32x4 p;
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        p[r] = d[r] * ((REV ? pair_decay(yhi[r], ylo[r], xhi, xlo) : pair_decay(xhi, xlo, yhi[r], ylo[r])) * a.pscale);
                    const bool masked = cut || yt == strip;
                    bool on[4] = {true, true, true, true};
                    if (masked) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            on[r] = takes<REV>(c, xt, y0 + r);
                            p[r] = on[r] ? p[r] : 0.0f;
                        }
                    }
                    if constexpr (MODE == kWalkDq) {
                        f32x4 d2 = {0, 0, 0, 0};
                        __builtin_amdgcn_sched_barrier(0);      // not both products' operands at once
#pragma unroll
                        for (int k = 0; k < VT; k += 2)
                            d2 = M::mma(M::transposed(l, sm.z + k * 16 * kC, yt), M::transposed(l, sm.z + (k + 1) * 16 * kC, yt),
                                        M::transposed(l, sm.e + k * 16 * kC, strip), M::transposed(l, sm.e + (k + 1) * 16 * kC, strip), d2);
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            cs[r] = on[r] ? p[r] * d2[r] : 0.0f;
                            rs += cs[r];
                        }
                    }
                    *pp = M::round(p);
                } else if (REV ? (strip & 1) && yt == strip - 1 : !(strip & 1) && yt == strip + 1) {
                    *pp = M::round(d);      // the other half of a step of 32 tokens
                }
                if constexpr (MODE == kWalkDq) {
                    store_sum16(l, &sm.csum[strip][yt * 16 + four], sum16(cs));
                }
            }
            if constexpr (MODE == kWalkDq) {
                rs += __shfl_xor(rs, 16);
                rs += __shfl_xor(rs, 32);
                if (l < 16) sm.rsum[ypart][xt] = rs;
            }
        }

        // x and the wave's part of the state that enters the chunk, for all tokens
        const bool bad = __builtin_amdgcn_readfirstlane(c.bad[0]) != 0;
        // the tokens whose out the wave finishes: all tiles of 16, or the first and the last, or the two between
        const auto own_tile = [&](int i) { return kParts == 1 ? i : part ? 1 + i : 3 * i; };
        f32x4 os[XT];
        {
            const int l = fresh<kTight>(lane_id());
            f32x4 all[4];
#pragma unroll
            for (int xt = 0; xt < 4; ++xt) all[xt] = f32x4{0, 0, 0, 0};
            const T* xs = sm.x + S.xf * kC;
#pragma unroll
            for (int k = 0; k < KF; k += 2) {
                Frag s0[NO], s1[NO];
                M::template split<NO>(S.s[k], s0);
                M::template split<NO>(S.s[k + 1], s1);
#pragma unroll
                for (int xt = 0; xt < 4; ++xt) {
                    const Frag f0 = M::transposed(l, xs + k * 16 * kC, xt), f1 = M::transposed(l, xs + (k + 1) * 16 * kC, xt);
#pragma unroll
                    for (int q = 0; q < NO; ++q) all[xt] = M::mma(f0, f1, s0[q], s1[q], all[xt]);
                }
            }
            if constexpr (kParts == 1) {
#pragma unroll
                for (int i = 0; i < XT; ++i) os[i] = all[i];
            } else {
                f32x4* half = sm.half + ((part ^ 1) * VT + ztile) * 2 * 64 + l;      // where the other part reads
                half[0] = part ? all[0] : all[1];
                half[64] = part ? all[3] : all[2];
                os[0] = part ? all[1] : all[0];
                os[1] = part ? all[2] : all[3];
            }
        }
        update<T, REV, NS>(S, sm.y, sm.z, c, cut, bad);
        __syncthreads();

        // out, from those sums and the chunk's own products
        {
            const int l = fresh<kTight>(lane_id()), col = l & 15, four = (l >> 4) * 4;
            Frag zf[4];
            const T* zt = sm.z + ztile * 16 * kC;
#pragma unroll
            for (int i = 0; i < 4; ++i) zf[i] = M::direct(l, zt, i);
            const int64_t t0 = (int64_t)chunk * kC;
#pragma unroll
            for (int i = 0; i < XT; ++i) {
                const int xt = own_tile(i), x0 = xt * 16 + four;
                f32x4 o = os[i];
                if constexpr (kParts == 2) o += sm.half[(w * 2 + i) * 64 + l];
                const f32x4 in = *reinterpret_cast<const f32x4*>(&c.in[x0]);
                o *= in;
                if (cut) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[r] = enters<REV>(c, x0 + r) ? o[r] : 0.0f;
                }
                if constexpr (MODE != kWalkPlain) {
                    f32x4 rd = o * M::widen(M::direct(l, sm.e + ztile * 16 * kC, xt));
                    if (cut) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) rd[r] = enters<REV>(c, x0 + r) ? rd[r] : 0.0f;
                    }
                    store_sum16(l, &sm.dot[ztile][x0], sum16(MODE == kWalkDk ? -rd : rd));
                }
                if (!bad) {
                    const T* pp = sm.p + xt * 16 * kC;
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        if (REV ? 2 * q + 1 >= xt : 2 * q <= xt)
                            o = M::mma(M::direct(l, pp, 2 * q), M::direct(l, pp, 2 * q + 1), zf[2 * q], zf[2 * q + 1], o);
                } else {
                    const int lb = here(l);
#pragma unroll 1
                    for (int y = 0; y < kC; ++y)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            if (takes<REV>(c, xt * 16 + (lb >> 4) * 4 + r, y))
                                o[r] = fmaf(tile_value(sm.p + xt * 16 * kC, (lb >> 4) * 4 + r, y), tile_value(zt, lb & 15, y), o[r]);
                        }
                }
                if (ztile * 16 + col < a.z.rows) {
                    TO* dst = op + col * L + t0 + x0;
                    if (t0 + x0 + 4 <= L) {
                        if constexpr (sizeof(TO) == 2) *reinterpret_cast<u32x2_a2*>(dst) = Mat<bf16_t>::round(o);
                        else *reinterpret_cast<u32x4_a4*>(dst) = __builtin_bit_cast(u32x4, o);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (t0 + x0 + r < L) Storage<TO>::store1(dst + r, o[r]);
                    }
                }
            }
        }
    }
    if constexpr (MODE != kWalkPlain) {
        __syncthreads();
        flush_r(begin + (n - 1) * step);
    }
    const bool ends = REV ? seg == 0 : seg == a.nseg - 1;       // the state leaves the row
    if constexpr (MODE == kWalkDq) {
        if (ends && a.bound_end) bound_store(a.nb);
    }
    if (ends && a.leave) S.store(a.leave + bh * sz, a);
}

// --------------------------------------------------------------------------------------------
// split rows: what each segment adds to the state (aggregate), then the states that enter the
// segments one after another (chain).  An aggregate is a walk without x and out and takes 0.4 to 0.55 of it
// (2 x 24 heads x 3001 tokens, dk 128, dv 64: 21 us of 38; the chain 7)
// --------------------------------------------------------------------------------------------
template <typename T, int KC, int VP>
struct AggSmem {
    __attribute__((aligned(16))) T y[KC * kC];
    __attribute__((aligned(16))) T z[VP * kC];
    ChunkDecay c[2];
};

template <typename T, int KC, int VP, bool REV, int NS>
__global__ __launch_bounds__((walk_threads(VP, walk_parts<T, KC, VP>()))) void walk_aggregate(WalkArgs a) {
    constexpr int VT = VP / 16, KF = KC / 16 / walk_parts<T, KC, VP>(), kThreads = walk_threads(VP, walk_parts<T, KC, VP>());
    __shared__ AggSmem<T, KC, VP> sm;
    const int l = lane_id(), w = wave_id();
    const int64_t L = a.seqlen;
    // the segment that nothing enters after it is left out
    const uint32_t id = walk_block((uint32_t)a.batch * a.heads * (a.nseg - 1));
    const uint32_t row = id / (uint32_t)(a.nseg - 1), bat = row / (uint32_t)a.heads;
    const int64_t bh = row, b = bat, h = row - bat * a.heads, seg = id - row * (a.nseg - 1) + (REV ? 1 : 0);
    const int chunks = (int)((L + kC - 1) / kC);
    const int first = (int)seg * a.seg_chunks, last = min(chunks, first + a.seg_chunks) - 1;
    const T* yp = head_base<T>(a.y, b, h, a.heads, L);
    const T* zp = head_base<T>(a.z, b, h, a.heads, L);
    State<KF> S;
    S.xf = w / VT * KF * 16;
    S.zf = w % VT * 16;
    S.load(nullptr, a);
    float all = 1.0f;
    TileRegs<T, KC, kThreads> yr;
    TileRegs<T, VP, kThreads> zr;
    constexpr int step = REV ? -1 : 1;
    const int begin = REV ? last : first, n = last - first + 1;
    if (threadIdx.x == 0) sm.c[0].bad[0] = sm.c[1].bad[0] = 0;
    TokenDecay td{0.0f, 1};
    if (w == 0) {
        td = load_decay(a, b, h, (int64_t)begin * kC + decay_token<REV>(l));
        chunk_decay<REV>(td, sm.c[0], a.iscale, a.uscale);
        if (n > 1) td = load_decay(a, b, h, (int64_t)(begin + step) * kC + decay_token<REV>(l));
    }
    const int tid = threadIdx.x;
    const auto load = [&](int chunk) {
        const uint32_t at = TileRegs<T, KC, kThreads>::offset_of(tid, chunk * kC, (int)L);
        yr.load(tid, at, yp, a.y.rows, (int)L);
        zr.load(tid, at, zp, a.z.rows, (int)L);
    };
    load(begin);
    for (int it = 0; it < n; ++it) {
        const int chunk = begin + it * step;
        ChunkDecay& c = sm.c[it & 1];
        __syncthreads();
        yr.settle(tid, yp, a.y.rows, (int64_t)chunk * kC, L);
        zr.settle(tid, zp, a.z.rows, (int64_t)chunk * kC, L);
        yr.store(tid, sm.y);
        zr.store(tid, sm.z);
        if (zr.zero_sum(yr.zero_sum(0.0f)) != 0.0f) c.bad[0] = 1;
        __syncthreads();
        if (it + 1 < n) {
            load(chunk + step);
            if (w == 0) {
                ChunkDecay& cn = sm.c[(it + 1) & 1];
                chunk_decay<REV>(td, cn, a.iscale, a.uscale);
                if (l == 0) cn.bad[0] = 0;
                if (it + 2 < n) td = load_decay(a, b, h, (int64_t)(chunk + 2 * step) * kC + decay_token<REV>(l));
            }
        }
        const bool cut = __builtin_amdgcn_readfirstlane(__float_as_int(c.a)) < 0;
        update<T, REV, NS>(S, sm.y, sm.z, c, cut, __builtin_amdgcn_readfirstlane(c.bad[0]) != 0);
        all = cut || all < 0.0f ? -1.0f : all * c.a;
    }
    const int64_t sz = (int64_t)a.x.rows * a.z.rows;
    S.store(a.seg + (bh * a.nseg + seg) * sz, a);
    if (threadIdx.x == 0) a.seg_a[bh * a.nseg + seg] = all;
}

// --------------------------------------------------------------------------------------------
// launches: one T, TO and KC in each translation unit
// --------------------------------------------------------------------------------------------
template <typename T, typename TO, int KC, int VP, int MODE, bool REV, int NS, int NO, int PARTS = walk_parts<T, KC, VP>()>
hipError_t launch_walk_one(const WalkArgs& a, hipStream_t s) {
    const int64_t blocks = (int64_t)a.batch * a.heads * a.nseg;
    hipLaunchKernelGGL((walk_kernel<T, TO, KC, VP, MODE, REV, NS, NO, PARTS>), dim3((unsigned)blocks),
                       dim3(walk_threads(VP, PARTS)), 0, s, a);
    return hipGetLastError();
}

template <typename T, typename TO, int KC, int VP, bool REV, int PARTS = walk_parts<T, KC, VP>()>
hipError_t launch_walk_plain(const WalkArgs& a, bool exact, hipStream_t s) {
    constexpr int kAll = Mat<T>::kSplit ? 3 : 1, kSome = Mat<T>::kSplit ? 2 : 1;
    return exact ? launch_walk_one<T, TO, KC, VP, kWalkPlain, REV, kAll, 1, PARTS>(a, s)
                 : launch_walk_one<T, TO, KC, VP, kWalkPlain, REV, kSome, 1, PARTS>(a, s);
}

template <typename T, typename TO, int KC, int VP>
hipError_t launch_walk_vp(const WalkArgs& a, WalkMode mode, bool exact, hipStream_t s) {
    constexpr int kAll = Mat<T>::kSplit ? 3 : 1;
    if (mode == kWalkDq) return launch_walk_one<T, TO, KC, VP, kWalkDq, false, kAll, kAll>(a, s);
    if (mode == kWalkDk) return launch_walk_one<T, TO, KC, VP, kWalkDk, true, kAll, kAll>(a, s);
    if constexpr (sizeof(T) == 2 && KC == 64 && VP == 64) {
        if ((int64_t)a.batch * a.heads * a.nseg >= kManyWalks)
            return a.rev ? launch_walk_plain<T, TO, KC, VP, true, 1>(a, exact, s)
                         : launch_walk_plain<T, TO, KC, VP, false, 1>(a, exact, s);
    }
    return a.rev ? launch_walk_plain<T, TO, KC, VP, true>(a, exact, s) : launch_walk_plain<T, TO, KC, VP, false>(a, exact, s);
}

template <typename T, typename TO, int KC>
hipError_t launch_walk_kc(const WalkArgs& a, WalkMode mode, bool exact, hipStream_t s) {
    return a.z.rows <= 64 ? launch_walk_vp<T, TO, KC, 64>(a, mode, exact, s)
                          : launch_walk_vp<T, TO, KC, 128>(a, mode, exact, s);
}

}  // namespace pm
