// gated_norm.hip -- the gated RMSNorm of (batch, dim, seqlen) activations, forward and backward: each group
// of consecutive features is normed by itself at every token, of a = x silu(z) (gate first) or of x, whose
// normed value silu(z) then multiplies.
//
// A block owns the features of one group at a tile of consecutive tokens: GROUPS lanes side by side, each with a
// 16-byte vector of tokens, and THREADS / GROUPS slices of the features.  A thread keeps what it
// read of its first KEPT features in registers from the sum over the features to the second sweep; features
// beyond those are read again.  Bound by HBM: three tensors in the forward, five in the backward.  8 x 4096
// tokens x 4096 features in 8 groups, bf16: forward 170 us (4.7 TB/s), backward 334 (4.0 TB/s, a copy 4.9; one block of
// 1024 threads a CU, whose loads, sum and stores follow each other, the VALU issuing 58% of the cycles).
#include "common.hpp"
#include "launch.hpp"
#include "linear.hpp"

namespace pm {
namespace {

// Offsets of a group's elements: 32 bits, added to a base that is the same for all lanes, where its bytes allow
// that (all but rows of 2^30 and more elements), else 64.  64-bit addresses of a thread's features took the
// registers of a whole feature's values.
template <bool FAR>
using Offset = std::conditional_t<FAR, int64_t, uint32_t>;
template <typename T, typename O>
__device__ __forceinline__ const T* at(const T* base, O off) {
    return reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + off * sizeof(T));
}
template <typename T, typename O>
__device__ __forceinline__ T* at(T* base, O off) {
    return reinterpret_cast<T*>(reinterpret_cast<char*>(base) + off * sizeof(T));
}
bool far(const GatedArgs& a) { return a.dim / a.groups * a.seqlen >= (int64_t)1 << 30; }

// The block's tile.  Blocks go to the 8 XCDs in turn; where rows end inside a line, neighbouring tiles share lines
// and are given to one XCD, an eighth of all tiles each, whose L2 then holds them (us, in turn and in eighths,
// forward and backward: 2 x 3001 x 1536 fp32 37, 55 against 28, 45; 8 x 4096 x 4096 bf16, whole lines, 169, 339
// against 180, 343), and so where a tile's piece of a row is less than a line (2 x 1024 x 4096 in tiles of 16 tokens 49,
// 87 against 30, 56).
template <typename T, int TILE>
__device__ __forceinline__ uint32_t tile_block(int64_t L) {
    const uint32_t id = blockIdx.x, per = gridDim.x / 8;
    return (TILE * sizeof(T) < 128 || L * (int64_t)sizeof(T) % 128) && id < per * 8 ? (id % 8) * per + id / 8 : id;
}

// The same raw values, unknown to the compiler: what it computed from them for the sum is computed again after it
// and not kept, which would take several times their registers.
template <typename T, int K>
__device__ __forceinline__ void forget(RawRun<T, K>& r) {
#pragma unroll
    for (int i = 0; i < RawRun<T, K>::kVecs; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t v = r.w[i][k];
            asm volatile("" : "+v"(v));
            r.w[i][k] = v;
        }
}

// The TOK tokens that a lane takes, from l0 on.  In rows of a vector and more (FULL) all loads are whole vectors: the one
// that would cross the row's end is read from further ahead, and lanes beyond the end read it too; a lane's own
// tokens are those from the own-th on.  Reading that vector's elements one by one, and its tile's features twice, made
// the row's last tile the last to end: 2 x 1001 x 4096 bf16, one group, 64 and 115 us, now 45 and 82.
template <int TOK>
struct Lane {
    int64_t l0;
    int own;
    __device__ Lane(int64_t L, int64_t t0, int grp) {
        const int64_t lt = t0 + grp * TOK;
        l0 = L >= TOK ? min(lt, L - TOK) : lt;
        own = L < TOK ? 0 : lt < L ? (int)(lt - l0) : TOK;
    }
    template <bool FULL, typename TO>
    __device__ __forceinline__ void store(TO* p, int64_t left, const float (&v)[TOK]) const {
        if constexpr (!FULL) {
            store_run<TO, TOK, false>(p, 0, left, v);
        } else if (own == 0) {
            store_run<TO, TOK, true>(p, 0, left, v);
        } else {
#pragma unroll
            for (int k = 1; k < TOK; ++k)
                if (k >= own) Storage<TO>::store1(p + k, v[k]);
        }
    }
};

// Sum over the slices of each token's value, in a fixed order; every thread gets its own tokens' sums.
template <int GROUPS, int THREADS, int TOK>
__device__ __forceinline__ void slices_sum(float (&v)[TOK], float (*red)[GROUPS * TOK], int grp) {
#pragma unroll
    for (int m = GROUPS; m < 64; m *= 2)
#pragma unroll
        for (int k = 0; k < TOK; ++k) v[k] += __shfl_xor(v[k], m);
    if ((int)(threadIdx.x & 63) < GROUPS) {
#pragma unroll
        for (int k = 0; k < TOK; ++k) red[threadIdx.x >> 6][grp * TOK + k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < TOK; ++k) v[k] = red[0][grp * TOK + k];
    for (int w = 1; w < THREADS / 64; ++w)
#pragma unroll
        for (int k = 0; k < TOK; ++k) v[k] += red[w][grp * TOK + k];
}

template <typename T, typename TO, int GROUPS, int THREADS, int KEPT, bool FIRST, bool FAR>
__global__ __launch_bounds__(THREADS) void gated_fwd_kernel(GatedArgs a) {
    constexpr int TOK = Storage<T>::kPerVec, SL = THREADS / GROUPS;
    __shared__ float red[THREADS / 64][GROUPS * TOK];
    const int grp = threadIdx.x % GROUPS, sl = threadIdx.x / GROUPS;
    const int64_t L = a.seqlen, tiles = (L + GROUPS * TOK - 1) / (GROUPS * TOK);
    const uint32_t id = tile_block<T, GROUPS * TOK>(L);
    const int64_t bg = id / (uint32_t)tiles, t0 = (id - bg * tiles) * (GROUPS * TOK);
    const int per = (int)(a.dim / a.groups);
    const Lane<TOK> lane(L, t0, grp);
    const int64_t l0 = lane.l0;
    const int64_t base = bg * per * L;
    const T* x = static_cast<const T*>(a.x) + base;
    const T* z = static_cast<const T*>(a.z) + base;
    TO* out = static_cast<TO*>(a.out) + base;
    const float* w = a.w + (bg % a.groups) * per;
    const auto body = [&](auto full_tag) {
        constexpr bool FULL = decltype(full_tag)::value;
        constexpr int C = FULL ? KEPT : 0;
        const int64_t left = L - l0;                            // tokens from the lane's first
        const auto off = [&](int f) { return (Offset<FAR>)f * (Offset<FAR>)L + (Offset<FAR>)l0; };
        RawRun<T, TOK> xr[KEPT], zr[KEPT];
        float kept[FIRST ? KEPT : 1][TOK];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            xr[i] = zr[i] = RawRun<T, TOK>{};
            const int f = sl + i * SL;
            if (f < per) {
                xr[i] = load_raw<T, TOK>(at(x, off(f)), 0);
                zr[i] = load_raw<T, TOK>(at(z, off(f)), 0);
            }
        }
        float s[TOK] = {};
        const auto value = [&](const float (&xv)[TOK], const float (&zv)[TOK], float (&v)[TOK]) {
#pragma unroll
            for (int k = 0; k < TOK; ++k) {
                v[k] = FIRST ? xv[k] * (zv[k] * sigmoid_f(zv[k])) : xv[k];
                s[k] = fmaf(v[k], v[k], s[k]);
            }
        };
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float xv[TOK], zv[TOK], v[TOK];
            unpack_run(xr[i], xv);
            unpack_run(zr[i], zv);
            value(xv, zv, v);
            if constexpr (FIRST) {
#pragma unroll
                for (int k = 0; k < TOK; ++k) kept[i][k] = v[k];
            }
        }
        for (int f = sl + C * SL; f < per; f += SL) {
            float xv[TOK], zv[TOK], v[TOK];
            load_run<T, TOK, FULL>(at(x, off(f)), 0, left, xv);
            if constexpr (FIRST) load_run<T, TOK, FULL>(at(z, off(f)), 0, left, zv);
            value(xv, zv, v);
        }
        slices_sum<GROUPS, THREADS, TOK>(s, red, grp);
        float r[TOK];
#pragma unroll
        for (int k = 0; k < TOK; ++k) r[k] = 1.0f / sqrtf(s[k] / (float)per + a.eps);
        if (sl == 0) {
#pragma unroll
            for (int k = 0; k < TOK; ++k)
                if (FULL ? k >= lane.own : l0 + k < L) a.rstd_out[bg * L + l0 + k] = r[k];
        }
        const auto put = [&](float (&v)[TOK], const float (&zv)[TOK], int f) {
            const float wv = w[f];
#pragma unroll
            for (int k = 0; k < TOK; ++k) {
                v[k] = v[k] * r[k] * wv;
                if constexpr (!FIRST) v[k] *= zv[k] * sigmoid_f(zv[k]);
            }
            lane.template store<FULL>(at(out, off(f)), left, v);
        };
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int f = sl + i * SL;
            float v[TOK], zv[TOK];
            if constexpr (FIRST) {
#pragma unroll
                for (int k = 0; k < TOK; ++k) v[k] = kept[i][k];
            } else {
                forget(xr[i]);
                unpack_run(xr[i], v);
                unpack_run(zr[i], zv);
            }
            if (f < per) put(v, zv, f);
        }
        for (int f = sl + C * SL; f < per; f += SL) {
            float v[TOK], zv[TOK];
            load_run<T, TOK, FULL>(at(x, off(f)), 0, left, v);
            load_run<T, TOK, FULL>(at(z, off(f)), 0, left, zv);
            if constexpr (FIRST) {
#pragma unroll
                for (int k = 0; k < TOK; ++k) v[k] *= zv[k] * sigmoid_f(zv[k]);
            }
            put(v, zv, f);
        }
    };
    if (L >= TOK) body(std::true_type{});
    else body(std::false_type{});
}

// The forward of single tokens (seqlen 1): a group's features are consecutive in memory, so the lanes take
// vectors of features.
template <typename T, typename TO, int THREADS, int KEPT, bool FIRST>
__global__ __launch_bounds__(THREADS) void gated_fwd_token(GatedArgs a) {
    constexpr int PV = Storage<T>::kPerVec;
    __shared__ float red[THREADS / 64];
    const int per = (int)(a.dim / a.groups);
    const int64_t bg = blockIdx.x, base = bg * per;
    const T* x = static_cast<const T*>(a.x) + base;
    const T* z = static_cast<const T*>(a.z) + base;
    TO* out = static_cast<TO*>(a.out) + base;
    const float* w = a.w + (bg % a.groups) * per;
    RawRun<T, PV> xr[KEPT], zr[KEPT];
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
        const int f = (threadIdx.x + i * THREADS) * PV;
        xr[i] = load_part<T, PV, false>(x, f, per);
        zr[i] = load_part<T, PV, false>(z, f, per);
    }
    float s = 0.0f;
    const auto value = [&](const RawRun<T, PV>& xw, const RawRun<T, PV>& zw, int f, float (&v)[PV], float (&gate)[PV]) {
        unpack_part<T, PV, false>(xw, x, f, per, v);
        unpack_part<T, PV, false>(zw, z, f, per, gate);
#pragma unroll
        for (int k = 0; k < PV; ++k) {
            gate[k] *= sigmoid_f(gate[k]);
            if constexpr (FIRST) v[k] *= gate[k];
        }
    };
    const auto sum = [&](const RawRun<T, PV>& xw, const RawRun<T, PV>& zw, int f) {
        float v[PV], gate[PV];
        value(xw, zw, f, v, gate);
#pragma unroll
        for (int k = 0; k < PV; ++k) s = fmaf(v[k], v[k], s);       // 0 beyond the group
    };
#pragma unroll
    for (int i = 0; i < KEPT; ++i) sum(xr[i], zr[i], (threadIdx.x + i * THREADS) * PV);
    for (int f = (threadIdx.x + KEPT * THREADS) * PV; f < per; f += THREADS * PV)
        sum(load_part<T, PV, false>(x, f, per), load_part<T, PV, false>(z, f, per), f);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) s += __shfl_xor(s, m);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    s = red[0];
#pragma unroll
    for (int i = 1; i < THREADS / 64; ++i) s += red[i];
    const float r = 1.0f / sqrtf(s / (float)per + a.eps);
    if (threadIdx.x == 0) a.rstd_out[bg] = r;
    const auto put = [&](const RawRun<T, PV>& xw, const RawRun<T, PV>& zw, int f) {
        if (f >= per) return;
        float v[PV], gate[PV], wv[PV];
        load_run<float, PV>(w, f, per, wv);
        value(xw, zw, f, v, gate);
#pragma unroll
        for (int k = 0; k < PV; ++k) {
            v[k] = v[k] * r * wv[k];
            if constexpr (!FIRST) v[k] *= gate[k];
        }
        store_run<TO, PV, false, false>(out, f, per, v);
    };
#pragma unroll
    for (int i = 0; i < KEPT; ++i) put(xr[i], zr[i], (threadIdx.x + i * THREADS) * PV);
    for (int f = (threadIdx.x + KEPT * THREADS) * PV; f < per; f += THREADS * PV)
        put(load_part<T, PV, false>(x, f, per), load_part<T, PV, false>(z, f, per), f);
}

// With up the gradient of a rstd (dout weight, or dout weight gate) and m the mean of up a over the group,
//   da = rstd (up - a rstd^2 m), and from it dx and dz; partial[b, tile, f] = the tile's sum for dweight.
// A tile has gated_tile() tokens, and partial a row for each.
template <typename T, typename TO, int GROUPS, int THREADS, int KEPT, bool FIRST, bool FAR>
__global__ __launch_bounds__(THREADS, (THREADS >= 512 ? 4 : THREADS / 128)) void gated_bwd_kernel(GatedArgs a) {
    constexpr int TOK = Storage<T>::kPerVec, SL = THREADS / GROUPS;
    __shared__ float red[THREADS / 64][GROUPS * TOK];
    const int grp = threadIdx.x % GROUPS, sl = threadIdx.x / GROUPS;
    constexpr int kTile = GROUPS * TOK;
    const int64_t L = a.seqlen, tiles = (L + kTile - 1) / kTile;
    const uint32_t id = tile_block<T, kTile>(L);
    const int64_t bg = id / (uint32_t)tiles, tile = id - bg * tiles, t0 = tile * kTile;
    const int64_t b = bg / a.groups;
    const int per = (int)(a.dim / a.groups), first = (int)(bg - b * a.groups) * per;
    const Lane<TOK> lane(L, t0, grp);
    const int64_t l0 = lane.l0;
    const int64_t base = bg * per * L;
    const T* x = static_cast<const T*>(a.x) + base;
    const T* z = static_cast<const T*>(a.z) + base;
    const T* g = static_cast<const T*>(a.dout) + base;
    TO* dx = static_cast<TO*>(a.out) + base;
    TO* dz = static_cast<TO*>(a.dz) + base;
    const float* w = a.w + first;
    float* part = a.partial + (b * tiles + tile) * a.dim + first;
    const auto body = [&](auto full_tag) {
        constexpr bool FULL = decltype(full_tag)::value;
        constexpr int C = FULL ? KEPT : 0;
        const int64_t left = L - l0;                            // tokens from the lane's first
        const auto off = [&](int f) { return (Offset<FAR>)f * (Offset<FAR>)L + (Offset<FAR>)l0; };
        RawRun<T, TOK> xr[KEPT], zr[KEPT], gr[KEPT];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            xr[i] = zr[i] = gr[i] = RawRun<T, TOK>{};
            const int f = sl + i * SL;
            if (f < per) {
                xr[i] = load_raw<T, TOK>(at(x, off(f)), 0);
                zr[i] = load_raw<T, TOK>(at(z, off(f)), 0);
                gr[i] = load_raw<T, TOK>(at(g, off(f)), 0);
            }
        }
        float s[TOK] = {};
        const auto dot = [&](const float (&xv)[TOK], const float (&zv)[TOK], const float (&gv)[TOK], float wv) {
#pragma unroll
            for (int k = 0; k < TOK; ++k) s[k] = fmaf(gv[k] * wv * (zv[k] * sigmoid_f(zv[k])), xv[k], s[k]);
        };
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float xv[TOK], zv[TOK], gv[TOK];
            unpack_run(xr[i], xv);
            unpack_run(zr[i], zv);
            unpack_run(gr[i], gv);
            const int f = sl + i * SL;
            if (f < per) dot(xv, zv, gv, w[f]);
            __builtin_amdgcn_sched_barrier(0);
        }
        for (int f = sl + C * SL; f < per; f += SL) {
            float xv[TOK], zv[TOK], gv[TOK];
            load_run<T, TOK, FULL>(at(x, off(f)), 0, left, xv);
            load_run<T, TOK, FULL>(at(z, off(f)), 0, left, zv);
            load_run<T, TOK, FULL>(at(g, off(f)), 0, left, gv);
            dot(xv, zv, gv, w[f]);
        }
        float r[TOK], c[TOK];
#pragma unroll
        for (int k = 0; k < TOK; ++k) r[k] = (FULL || l0 + k < L) ? a.rstd[bg * L + l0 + k] : 0.0f;
        slices_sum<GROUPS, THREADS, TOK>(s, red, grp);
#pragma unroll
        for (int k = 0; k < TOK; ++k) c[k] = r[k] * r[k] * (s[k] / (float)per);
        const auto grad = [&](const float (&xv)[TOK], const float (&zv)[TOK], const float (&gv)[TOK], int f) {
            const float wv = w[f];
            float ox[TOK], oz[TOK], pw = 0.0f;
#pragma unroll
            for (int k = 0; k < TOK; ++k) {
                const float sig = sigmoid_f(zv[k]), gate = zv[k] * sig, dgate = sig * fmaf(zv[k], 1.0f - sig, 1.0f);
                if constexpr (FIRST) {
                    const float av = xv[k] * gate, da = r[k] * (gv[k] * wv - av * c[k]);
                    ox[k] = da * gate;
                    oz[k] = da * xv[k] * dgate;
                    pw = k >= lane.own ? fmaf(gv[k] * av, r[k], pw) : pw;
                } else {
                    ox[k] = r[k] * (gv[k] * wv * gate - xv[k] * c[k]);
                    const float n = gv[k] * xv[k] * r[k];
                    oz[k] = n * wv * dgate;
                    pw = k >= lane.own ? fmaf(n, gate, pw) : pw;
                }
            }
            lane.template store<FULL>(at(dx, off(f)), left, ox);
            lane.template store<FULL>(at(dz, off(f)), left, oz);
#pragma unroll
            for (int m = 1; m < GROUPS; m *= 2) pw += __shfl_xor(pw, m, GROUPS);
            if (grp == 0) part[f] = pw;
        };
#pragma unroll
        for (int i = 0; i < C; ++i) {
            forget(xr[i]);
            forget(zr[i]);
            forget(gr[i]);
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float xv[TOK], zv[TOK], gv[TOK];
            unpack_run(xr[i], xv);
            unpack_run(zr[i], zv);
            unpack_run(gr[i], gv);
            const int f = sl + i * SL;
            if (f < per) grad(xv, zv, gv, f);
            __builtin_amdgcn_sched_barrier(0);          // one feature's values at a time
        }
        for (int f = sl + C * SL; f < per; f += SL) {
            float xv[TOK], zv[TOK], gv[TOK];
            load_run<T, TOK, FULL>(at(x, off(f)), 0, left, xv);
            load_run<T, TOK, FULL>(at(z, off(f)), 0, left, zv);
            load_run<T, TOK, FULL>(at(g, off(f)), 0, left, gv);
            grad(xv, zv, gv, f);
        }
    };
    if (L >= TOK) body(std::true_type{});
    else body(std::false_type{});
}

template <typename T, typename TO, int GROUPS, int THREADS, int KEPT, bool FIRST>
hipError_t fwd_one(const GatedArgs& a, hipStream_t s) {
    constexpr int64_t kTile = GROUPS * Storage<T>::kPerVec;
    const int64_t blocks = a.batch * a.groups * ((a.seqlen + kTile - 1) / kTile);
    if (far(a))
        hipLaunchKernelGGL((gated_fwd_kernel<T, TO, GROUPS, THREADS, KEPT, FIRST, true>), dim3((unsigned)blocks), dim3(THREADS), 0, s, a);
    else
        hipLaunchKernelGGL((gated_fwd_kernel<T, TO, GROUPS, THREADS, KEPT, FIRST, false>), dim3((unsigned)blocks), dim3(THREADS), 0, s, a);
    return hipGetLastError();
}

template <typename T, typename TO, int THREADS, int KEPT, bool FIRST>
hipError_t token_one(const GatedArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((gated_fwd_token<T, TO, THREADS, KEPT, FIRST>), dim3((unsigned)(a.batch * a.groups)), dim3(THREADS), 0, s, a);
    return hipGetLastError();
}

// Threads of a block: slices that leave a thread about as many features as it keeps.  Us of the bf16 forward and
// backward of 2 x 4096 tokens with 256, 512 and 1024 threads (features of a group):
//   2048 in groups of 128 24, 38, 91; 35, 40, 61   of 256 19, 24, 51; 37, 36, 47   4096 in groups of 512 41, 34, 58; 76, 72, 74
//   4096 in one 130, 72, 62; 219, 126, 97          fp32 backward, 2048 in groups of 256 75, 66, 60
// Single tokens with 64 and 512: 64 x 4096 in groups of 512 3.8, 5.2, of 768 4.0, 4.1, in one 8.4, 4.2.  Tiles of 8 tokens
// with 256 and 1024: 64 rows of 4 x 4096 in groups of 512 10.1, 14.2, of 1024 12.5, 10.2; tiles of 16: 256 tokens in groups of
// 512 8.0, 11.4, of 4096 30, 19.
template <typename T, typename TO, bool FIRST>
hipError_t fwd_t(const GatedArgs& a, hipStream_t s) {
    constexpr int kFew = (int)kGatedFewTokens / Storage<T>::kPerVec, kNarrow = (int)kGatedNarrow / Storage<T>::kPerVec;
    const int64_t per = a.dim / a.groups, tile = gated_tile(a.batch, a.seqlen, a.groups);
    if (a.seqlen == 1) return per <= 512 ? token_one<T, TO, 64, 2, FIRST>(a, s) : token_one<T, TO, 512, 2, FIRST>(a, s);
    if (tile == kGatedFewTokens)
        return per <= 512 ? fwd_one<T, TO, kFew, 256, 2, FIRST>(a, s) : fwd_one<T, TO, kFew, 1024, 4, FIRST>(a, s);
    if (tile == kGatedNarrow)
        return per <= 512 ? fwd_one<T, TO, kNarrow, 256, 4, FIRST>(a, s) : fwd_one<T, TO, kNarrow, 1024, 4, FIRST>(a, s);
    if (per <= 256) return fwd_one<T, TO, 8, 256, 8, FIRST>(a, s);
    if (per <= 512) return fwd_one<T, TO, 8, 512, 8, FIRST>(a, s);
    return fwd_one<T, TO, 8, 1024, 8, FIRST>(a, s);
}

template <typename T, typename TO, int GROUPS, int THREADS, int KEPT, bool FIRST>
hipError_t bwd_one(const GatedArgs& a, hipStream_t s) {
    constexpr int64_t kTile = GROUPS * Storage<T>::kPerVec;
    const int64_t tiles = (a.seqlen + kTile - 1) / kTile;
    const dim3 grid((unsigned)(a.batch * a.groups * tiles));
    if (far(a)) hipLaunchKernelGGL((gated_bwd_kernel<T, TO, GROUPS, THREADS, KEPT, FIRST, true>), grid, dim3(THREADS), 0, s, a);
    else hipLaunchKernelGGL((gated_bwd_kernel<T, TO, GROUPS, THREADS, KEPT, FIRST, false>), grid, dim3(THREADS), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
    return launch_partial_rows_sum(a.partial, a.dw, a.batch * tiles, a.dim, s);
}

template <typename T, typename TO, bool FIRST>
hipError_t bwd_t(const GatedArgs& a, hipStream_t s) {
    constexpr int TOK = Storage<T>::kPerVec, kWide = (int)kRmsTile / TOK;
    constexpr int kFew = (int)kGatedFewTokens / TOK, kNarrow = (int)kGatedNarrow / TOK;
    const int64_t per = a.dim / a.groups, tile = gated_tile(a.batch, a.seqlen, a.groups);
    if (tile == kGatedFewTokens)
        return per <= 512 ? bwd_one<T, TO, kFew, 256, 2, FIRST>(a, s) : bwd_one<T, TO, kFew, 1024, 4, FIRST>(a, s);
    if (tile == kGatedNarrow)
        return per <= 512 ? bwd_one<T, TO, kNarrow, 256, 4, FIRST>(a, s) : bwd_one<T, TO, kNarrow, 1024, 4, FIRST>(a, s);
    if (per <= 128) return bwd_one<T, TO, kWide, 256, 4, FIRST>(a, s);
    if (per <= 256) return bwd_one<T, TO, kWide, 512, 4, FIRST>(a, s);
    return bwd_one<T, TO, kWide, 1024, 4, FIRST>(a, s);
}

template <bool FIRST>
hipError_t fwd_d(const GatedArgs& a, hipStream_t s) {
    switch (a.dtype) {
        case 1: return fwd_t<bf16_t, bf16_t, FIRST>(a, s);
        case 2: return fwd_t<bf16_t, float, FIRST>(a, s);
        default: return fwd_t<float, float, FIRST>(a, s);
    }
}
template <bool FIRST>
hipError_t bwd_d(const GatedArgs& a, hipStream_t s) {
    switch (a.dtype) {
        case 1: return bwd_t<bf16_t, bf16_t, FIRST>(a, s);
        case 2: return bwd_t<bf16_t, float, FIRST>(a, s);
        default: return bwd_t<float, float, FIRST>(a, s);
    }
}

}  // namespace

hipError_t launch_gated_fwd(const GatedArgs& a, hipStream_t s) { return a.gate_first ? fwd_d<true>(a, s) : fwd_d<false>(a, s); }
hipError_t launch_gated_bwd(const GatedArgs& a, hipStream_t s) { return a.gate_first ? bwd_d<true>(a, s) : bwd_d<false>(a, s); }

}  // namespace pm
