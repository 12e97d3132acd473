// norms.hip -- norms over the features of (rows, dim, seqlen) activations, token by token, forward and backward:
//   layer norm     h = (x - mean) r,  r = 1 / sqrt(var + eps),  out = h w + b
//                  dx = r (g w - mean(g w) - h mean(g w h)) (+ dres),  dw = sum g h,  db = sum g
//   head's length  out = x r,  r = 1 / sqrt(sum x^2 + eps);   dx = r (g - x r^2 sum(x g))
// A block owns a tile of consecutive tokens of one row: LANES lanes side by side, each with one 16-byte vector of
// tokens, and THREADS / LANES slices of the features.  A thread keeps the vectors of its first KEPT features in registers
// from the sums to the second sweep; features beyond those are read again.  The variance takes one sweep: a
// thread sums its features' differences from its first one, and their squares, which loses nothing to a large mean;
// then mean and the squares about it are put together from the threads' own.
// Bound by HBM where there are tiles enough for the GPU; the layer norm's backward holds half of 2048 features and reads
// the others twice, with one block a CU, whose loads and stores take turns.  Us (a copy of 1 GiB runs at 5.2 TB/s):
//   layer norm  8 x 2048 x 4096 bf16: forward 72 (268 MB, 3.7 TB/s), backward with a residual 144 (537 MB, 3.7 TB/s); fp32 124, 243
//   length      8 x 2048 (16 heads) x 4096 bf16: backward 74 (405 MB, 5.5 TB/s); 2 x 1536 (24) x 3001 fp32: forward 18
#include "common.hpp"
#include "norms.hpp"

namespace pm {
namespace {

enum NormKind : int { kLayer = 0, kLength = 1 };

template <int LANES, int THREADS, int N>
struct SumSmem {
    __attribute__((aligned(16))) float red[THREADS / 64][LANES * N];
    __attribute__((aligned(16))) float tot[LANES * N];
};

// The sums over the slices of each lane's N values, in a fixed order, to every thread.
template <int LANES, int THREADS, int N>
__device__ __forceinline__ void slice_sums(float (&v)[N], SumSmem<LANES, THREADS, N>& sm) {
    const int l = threadIdx.x & 63, lane = threadIdx.x % LANES, w = threadIdx.x / 64;
#pragma unroll
    for (int m = LANES; m < 64; m *= 2)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor(v[k], m);
    if (l < LANES) {
#pragma unroll
        for (int k = 0; k < N; k += 4) *reinterpret_cast<f32x4*>(&sm.red[w][lane * N + k]) = f32x4{v[k], v[k + 1], v[k + 2], v[k + 3]};
    }
    __syncthreads();
    if (threadIdx.x < LANES * N) {
        float s = sm.red[0][threadIdx.x];
#pragma unroll
        for (int i = 1; i < THREADS / 64; ++i) s += sm.red[i][threadIdx.x];
        sm.tot[threadIdx.x] = s;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; k += 4) {
        const f32x4 t = *reinterpret_cast<const f32x4*>(&sm.tot[lane * N + k]);
        v[k] = t.x; v[k + 1] = t.y; v[k + 2] = t.z; v[k + 3] = t.w;
    }
}

// The block's tile.  Blocks go to the 8 XCDs in turn: of 64 blocks each XCD takes eight tiles that follow each other, which share
// lines of 128 bytes where tiles are narrower or rows end inside one.  Us of the backward (batch x features x tokens) with
// this, as they come, and with each XCD's tiles all together, which leaves some memory channels idle: layer norm, bf16
// 8 x 2048 x 4096 144, 146, 159, x 4001 188, 236, 204; length 8 x 2048 x 4096 74, 82, 83; fp32 forward 2 x 1536 x 3001 18, 22, 19.
__device__ __forceinline__ int64_t norm_tile() {
    const uint32_t id = blockIdx.x, g = id / 64 * 64, r = id - g;
    return g + 64 > gridDim.x ? id : g + (r % 8) * 8 + r / 8;
}

template <typename T, typename TO, int KIND, int LANES, int THREADS, int KEPT>
__global__ __launch_bounds__(THREADS) void norm_fwd_kernel(NormArgs a) {
    constexpr int TOK = Storage<T>::kPerVec, SL = THREADS / LANES, kTile = LANES * TOK;
    __shared__ SumSmem<LANES, THREADS, TOK> sm;
    const int lane = threadIdx.x % LANES, sl = threadIdx.x / LANES;
    const int64_t L = a.seqlen, dim = a.dim, tiles = (L + kTile - 1) / kTile, id = norm_tile();
    const int64_t row = id / tiles, t0 = (id - row * tiles) * kTile;
    const bool whole = t0 + kTile <= L || L % TOK == 0;          // no vector crosses the row end
    const bool live = t0 + lane * TOK < L;
    const int64_t l0 = whole && !live ? t0 : t0 + lane * TOK;
    const T* xb = static_cast<const T*>(a.x) + row * dim * L;
    TO* ob = static_cast<TO*>(a.out) + row * dim * L;
    // FULL (block-uniform): lanes past the row end repeat the tile's first and store nothing
    const auto body = [&](auto full_tag) {
        constexpr bool FULL = decltype(full_tag)::value;
        constexpr int C = FULL ? KEPT : 0;
        RawRun<T, TOK> xr[KEPT];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            xr[i] = RawRun<T, TOK>{};
            if (sl + i * SL < dim) xr[i] = load_raw<T, TOK>(xb + (sl + (int64_t)i * SL) * L, l0);
        }
        float first[TOK], s[TOK] = {}, sq[TOK] = {};
        const auto take = [&](const float (&v)[TOK]) {
#pragma unroll
            for (int k = 0; k < TOK; ++k) {
                const float d = KIND == kLayer ? v[k] - first[k] : v[k];
                if (KIND == kLayer) s[k] += d;
                sq[k] = fmaf(d, d, sq[k]);
            }
        };
#pragma unroll
        for (int k = 0; k < TOK; ++k) first[k] = 0.0f;
        if constexpr (KIND == kLayer) {
            if constexpr (C > 0) unpack_run(xr[0], first);
            else if (sl < dim) load_run<T, TOK, FULL>(xb + (int64_t)sl * L, l0, L, first);
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float v[TOK];
            unpack_run(xr[i], v);
            if (sl + i * SL < dim) take(v);
        }
        for (int64_t f = sl + (int64_t)C * SL; f < dim; f += SL) {
            float v[TOK];
            load_run<T, TOK, FULL>(xb + f * L, l0, L, v);
            take(v);
        }
        float mean[TOK], r[TOK];
        if constexpr (KIND == kLayer) {
            const float n = sl < dim ? (float)((dim - sl + SL - 1) / SL) : 0.0f, inv = n > 0.0f ? 1.0f / n : 0.0f;
            float own[TOK];
#pragma unroll
            for (int k = 0; k < TOK; ++k) {
                own[k] = fmaf(s[k], inv, first[k]);              // the thread's mean, and its squares about it
                sq[k] = n > 0.0f ? fmaf(-s[k] * inv, s[k], sq[k]) : 0.0f;
                mean[k] = n * own[k];
            }
            slice_sums<LANES, THREADS, TOK>(mean, sm);
#pragma unroll
            for (int k = 0; k < TOK; ++k) {
                mean[k] /= (float)dim;
                const float d = own[k] - mean[k];
                if (n > 0.0f) sq[k] = fmaf(n * d, d, sq[k]);
            }
            __syncthreads();
        }
        slice_sums<LANES, THREADS, TOK>(sq, sm);
#pragma unroll
        for (int k = 0; k < TOK; ++k) r[k] = 1.0f / sqrtf((KIND == kLayer ? sq[k] / (float)dim : sq[k]) + a.eps);
        if (sl == 0) {
#pragma unroll
            for (int k = 0; k < TOK; ++k)
                if (FULL ? live : l0 + k < L) {
                    a.rstd_out[row * L + l0 + k] = r[k];
                    if (KIND == kLayer) a.mean_out[row * L + l0 + k] = mean[k];
                }
        }
        const auto write = [&](float (&v)[TOK], int64_t f) {
            const float wv = KIND == kLayer ? a.w[f] : 1.0f, bv = KIND == kLayer && a.b ? a.b[f] : 0.0f;
#pragma unroll
            for (int k = 0; k < TOK; ++k) v[k] = KIND == kLayer ? fmaf((v[k] - mean[k]) * r[k], wv, bv) : v[k] * r[k];
            if constexpr (FULL) { if (live) store_run<TO, TOK, true>(ob + f * L, l0, L, v); }
            else store_run<TO, TOK>(ob + f * L, l0, L, v);
        };
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float v[TOK];
            unpack_run(xr[i], v);
            if (sl + i * SL < dim) write(v, sl + (int64_t)i * SL);
        }
        for (int64_t f = sl + (int64_t)C * SL; f < dim; f += SL) {
            float v[TOK];
            load_run<T, TOK, FULL>(xb + f * L, l0, L, v);
            write(v, f);
        }
    };
    if (whole) body(std::true_type{});
    else body(std::false_type{});
}

// Layer norm: partial[tile, 0, f] and [tile, 1, f] are the tile's sums of g h and g.
template <typename T, typename TO, int KIND, int LANES, int THREADS, int KEPT>
__global__ __launch_bounds__(THREADS) void norm_bwd_kernel(NormArgs a) {
    constexpr int TOK = Storage<T>::kPerVec, SL = THREADS / LANES, kTile = LANES * TOK, N = KIND == kLayer ? 2 * TOK : TOK;
    __shared__ SumSmem<LANES, THREADS, N> sm;
    const int lane = threadIdx.x % LANES, sl = threadIdx.x / LANES;
    const int64_t L = a.seqlen, dim = a.dim, tiles = (L + kTile - 1) / kTile, id = norm_tile();
    const int64_t row = id / tiles, t0 = (id - row * tiles) * kTile;
    const bool whole = t0 + kTile <= L || L % TOK == 0;
    const bool live = t0 + lane * TOK < L;
    const int64_t l0 = whole && !live ? t0 : t0 + lane * TOK;
    const int64_t off = row * dim * L;
    const T* xb = static_cast<const T*>(a.x) + off;
    const T* gb = static_cast<const T*>(a.dout) + off;
    const T* rb = static_cast<const T*>(a.dres);
    if (rb) rb += off;
    TO* ob = static_cast<TO*>(a.out) + off;
    const auto body = [&](auto full_tag) {
        constexpr bool FULL = decltype(full_tag)::value;
        constexpr int C = FULL ? KEPT : 0;
        RawRun<T, TOK> xr[KEPT], gr[KEPT];
#pragma unroll
        for (int i = 0; i < C; ++i) {
            xr[i] = gr[i] = RawRun<T, TOK>{};
            if (sl + i * SL < dim) {
                xr[i] = load_raw<T, TOK>(xb + (sl + (int64_t)i * SL) * L, l0);
                gr[i] = load_raw<T, TOK>(gb + (sl + (int64_t)i * SL) * L, l0);
            }
        }
        float mean[TOK], r[TOK], s[N] = {};
#pragma unroll
        for (int k = 0; k < TOK; ++k) {
            const bool in = FULL || l0 + k < L;
            r[k] = in ? a.rstd[row * L + l0 + k] : 0.0f;
            mean[k] = KIND == kLayer && in ? a.mean[row * L + l0 + k] : 0.0f;
        }
        const auto take = [&](const float (&x)[TOK], const float (&g)[TOK], int64_t f) {
            const float wv = KIND == kLayer ? a.w[f] : 1.0f;
#pragma unroll
            for (int k = 0; k < TOK; ++k) {
                if constexpr (KIND == kLayer) {
                    const float gw = g[k] * wv;
                    s[k] += gw;
                    s[TOK + k] = fmaf(gw, (x[k] - mean[k]) * r[k], s[TOK + k]);
                } else {
                    s[k] = fmaf(g[k], x[k], s[k]);
                }
            }
        };
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float x[TOK], g[TOK];
            unpack_run(xr[i], x);
            unpack_run(gr[i], g);
            if (sl + i * SL < dim) take(x, g, sl + (int64_t)i * SL);
        }
        for (int64_t f = sl + (int64_t)C * SL; f < dim; f += SL) {
            float x[TOK], g[TOK];
            load_run<T, TOK, FULL>(xb + f * L, l0, L, x);
            load_run<T, TOK, FULL>(gb + f * L, l0, L, g);
            take(x, g, f);
        }
        slice_sums<LANES, THREADS, N>(s, sm);
        float c1[TOK], c2[TOK];
#pragma unroll
        for (int k = 0; k < TOK; ++k) {
            c1[k] = KIND == kLayer ? s[k] / (float)dim : 0.0f;
            c2[k] = KIND == kLayer ? s[N - TOK + k] / (float)dim : s[k] * r[k] * r[k];
        }
        const auto grad = [&](const float (&x)[TOK], const float (&g)[TOK], int64_t f) {
            const float wv = KIND == kLayer ? a.w[f] : 1.0f;
            float o[TOK], pw = 0.0f, pb = 0.0f;
            if (KIND == kLayer && rb) load_run<T, TOK, FULL>(rb + f * L, l0, L, o);
            else {
#pragma unroll
                for (int k = 0; k < TOK; ++k) o[k] = 0.0f;
            }
#pragma unroll
            for (int k = 0; k < TOK; ++k) {
                if constexpr (KIND == kLayer) {
                    const float h = (x[k] - mean[k]) * r[k];
                    o[k] += r[k] * (g[k] * wv - c1[k] - h * c2[k]);
                    pw = fmaf(g[k], h, pw);                      // 0 past the row end: g reads 0 there
                    pb += g[k];
                } else {
                    o[k] = r[k] * (g[k] - x[k] * c2[k]);
                }
            }
            if constexpr (FULL) { if (live) store_run<TO, TOK, true>(ob + f * L, l0, L, o); }
            else store_run<TO, TOK>(ob + f * L, l0, L, o);
            if constexpr (KIND == kLayer) {
                if (FULL && !live) pw = pb = 0.0f;
#pragma unroll
                for (int m = 1; m < LANES; m *= 2) {
                    pw += __shfl_xor(pw, m, LANES);
                    pb += __shfl_xor(pb, m, LANES);
                }
                if (lane == 0) {
                    a.partial[id * 2 * dim + f] = pw;
                    a.partial[(id * 2 + 1) * dim + f] = pb;
                }
            }
        };
#pragma unroll
        for (int i = 0; i < C; ++i) {
            float x[TOK], g[TOK];
            unpack_run(xr[i], x);
            unpack_run(gr[i], g);
            if (sl + i * SL < dim) grad(x, g, sl + (int64_t)i * SL);
        }
        for (int64_t f = sl + (int64_t)C * SL; f < dim; f += SL) {
            float x[TOK], g[TOK];
            load_run<T, TOK, FULL>(xb + f * L, l0, L, x);
            load_run<T, TOK, FULL>(gb + f * L, l0, L, g);
            grad(x, g, f);
        }
    };
    if (whole) body(std::true_type{});
    else body(std::false_type{});
}

// dweight and dbias from the tiles' sums, in a fixed order: a block owns 32 of the 2 dim columns, each of its 32 row groups
// sums every 32nd row, eight loads in flight, and the groups' sums are added in order.
constexpr int kFinCols = 32, kFinRows = 32;
__global__ __launch_bounds__(kFinCols * kFinRows) void norm_partial_sums(const float* __restrict__ partial, float* __restrict__ dw,
                                                                         float* __restrict__ db, int64_t rows, int64_t dim) {
    __shared__ float part[kFinRows][kFinCols];
    const int co = threadIdx.x % kFinCols, rg = threadIdx.x / kFinCols;
    const int64_t f = (int64_t)blockIdx.x * kFinCols + co, cols = 2 * dim;
    float v = 0.0f;
    if (f < cols) {
        int64_t i = rg;
        for (; i + 7 * kFinRows < rows; i += 8 * kFinRows) {
            float w[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) w[q] = partial[(i + q * kFinRows) * cols + f];
            v += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
        }
        for (; i < rows; i += kFinRows) v += partial[i * cols + f];
    }
    part[rg][co] = v;
    __syncthreads();
    if (rg == 0 && f < cols) {
#pragma unroll
        for (int q = 1; q < kFinRows; ++q) v += part[q][co];
        if (f < dim) dw[f] = v;
        else if (db) db[f - dim] = v;
    }
}

// Rows of one token: their features are consecutive.  A row to GROUP threads, in vectors; the sums as above.
template <typename T, typename TO, int KIND, int GROUP>
__global__ __launch_bounds__(256) void norm_token_kernel(NormArgs a) {
    constexpr int PER = Storage<T>::kPerVec, kWaves = GROUP / 64 > 0 ? GROUP / 64 : 1, KEPT = 4;
    __shared__ float red[2][kWaves];
    const int64_t row = (int64_t)blockIdx.x * (256 / GROUP) + threadIdx.x / GROUP, dim = a.dim;
    const int g = threadIdx.x % GROUP;
    if (row >= a.rows) return;                           // whole waves, and GROUP 256 has no such row
    const T* x = static_cast<const T*>(a.x) + row * dim;
    TO* o = static_cast<TO*>(a.out) + row * dim;
    const auto sum = [&](float v, int which) {
#pragma unroll
        for (int m = 1; m < (GROUP < 64 ? GROUP : 64); m *= 2) v += __shfl_xor(v, m);
        if constexpr (GROUP > 64) {
            if ((threadIdx.x & 63) == 0) red[which][threadIdx.x / 64] = v;
            __syncthreads();
            v = red[which][0];
#pragma unroll
            for (int i = 1; i < kWaves; ++i) v += red[which][i];
        }
        return v;
    };
    float kept[KEPT][PER];
    float first = 0.0f, s = 0.0f, sq = 0.0f, n = 0.0f;
    bool any = false;
    const auto take = [&](const float (&v)[PER], int count) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (k >= count) break;
            if (KIND == kLayer && !any) first = v[k];
            any = true;
            const float d = KIND == kLayer ? v[k] - first : v[k];
            if (KIND == kLayer) s += d;
            sq = fmaf(d, d, sq);
            n += 1.0f;
        }
    };
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
        const int64_t f = ((int64_t)i * GROUP + g) * PER;
        load_run<T, PER>(x, f < dim ? f : dim, dim, kept[i]);
    }
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
        const int64_t f = ((int64_t)i * GROUP + g) * PER;
        take(kept[i], (int)min((int64_t)PER, max((int64_t)0, dim - f)));
    }
    for (int64_t f = ((int64_t)KEPT * GROUP + g) * PER; f < dim; f += GROUP * PER) {
        float v[PER];
        load_run<T, PER>(x, f, dim, v);
        take(v, (int)min((int64_t)PER, dim - f));
    }
    float mean = 0.0f;
    if constexpr (KIND == kLayer) {
        const float inv = n > 0.0f ? 1.0f / n : 0.0f, own = fmaf(s, inv, first);
        mean = sum(n * own, 0) / (float)dim;
        const float d = own - mean;
        sq = n > 0.0f ? fmaf(n * d, d, fmaf(-s * inv, s, sq)) : 0.0f;
    }
    sq = sum(sq, 1);
    const float r = 1.0f / sqrtf((KIND == kLayer ? sq / (float)dim : sq) + a.eps);
    if (g == 0) {
        a.rstd_out[row] = r;
        if (KIND == kLayer) a.mean_out[row] = mean;
    }
    const auto write = [&](float (&v)[PER], int64_t f) {
        if (KIND == kLayer) {
            float w[PER], b[PER];
#pragma unroll
            for (int k = 0; k < PER; k += 4) {
                load_run<float, 4>(a.w, f + k < dim ? f + k : dim, dim, w + k);
                if (a.b) load_run<float, 4>(a.b, f + k < dim ? f + k : dim, dim, b + k);
            }
#pragma unroll
            for (int k = 0; k < PER; ++k) v[k] = fmaf((v[k] - mean) * r, w[k], a.b ? b[k] : 0.0f);
        } else {
#pragma unroll
            for (int k = 0; k < PER; ++k) v[k] *= r;
        }
        store_run<TO, PER>(o, f, dim, v);
    };
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
        const int64_t f = ((int64_t)i * GROUP + g) * PER;
        if (f < dim) write(kept[i], f);
    }
    for (int64_t f = ((int64_t)KEPT * GROUP + g) * PER; f < dim; f += GROUP * PER) {
        float v[PER];
        load_run<T, PER>(x, f, dim, v);
        write(v, f);
    }
}

template <typename T, typename TO, int KIND, int LANES, int THREADS, int KEPT>
hipError_t fwd_one(const NormArgs& a, hipStream_t s) {
    constexpr int64_t kTile = LANES * Storage<T>::kPerVec;
    hipLaunchKernelGGL((norm_fwd_kernel<T, TO, KIND, LANES, THREADS, KEPT>), dim3((unsigned)(a.rows * ((a.seqlen + kTile - 1) / kTile))),
                       dim3(THREADS), 0, s, a);
    return hipGetLastError();
}
template <typename T, typename TO, int KIND, int LANES, int THREADS, int KEPT>
hipError_t bwd_one(const NormArgs& a, hipStream_t s) {
    constexpr int64_t kTile = LANES * Storage<T>::kPerVec;
    hipLaunchKernelGGL((norm_bwd_kernel<T, TO, KIND, LANES, THREADS, KEPT>), dim3((unsigned)(a.rows * ((a.seqlen + kTile - 1) / kTile))),
                       dim3(THREADS), 0, s, a);
    return hipGetLastError();
}

// 64 threads a row or 256.  Us of the layer norm: 64 x 512 4.0, 4.3; 64 x 768 4.9, 4.5.
template <typename T, typename TO, int KIND>
hipError_t token_t(const NormArgs& a, hipStream_t s) {
    if (a.dim <= 64 * Storage<T>::kPerVec)
        hipLaunchKernelGGL((norm_token_kernel<T, TO, KIND, 64>), dim3((unsigned)((a.rows + 3) / 4)), dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((norm_token_kernel<T, TO, KIND, 256>), dim3((unsigned)a.rows), dim3(256), 0, s, a);
    return hipGetLastError();
}

// Threads of a layer norm's block by its features, many with more of them kept or few.  Us (batch x features x tokens, bf16;
// forward, backward) with 1024 threads and with 256, tiles of 128 bytes: 8 x 256 x 4096 17, 23 and 9.6, 16; x 512 21, 32 and
// 17, 33; x 768 26, 40 and 29, 43.  With 1024 and with 512, tiles of 64 bytes: 4 x 512 x 2048 9.8, 13 and 8.0, 11; x 768 11, 15
// and 9.1, 14.
constexpr int64_t kFew8 = 512, kFew4 = 768;
template <typename T, typename TO>
hipError_t layer_fwd_t(const NormArgs& a, hipStream_t s) {
    if (a.seqlen == 1) return token_t<T, TO, kLayer>(a, s);
    switch (norm_lanes(a.rows, a.seqlen, sizeof(T) == 4)) {
        case 1: return fwd_one<T, TO, kLayer, 1, 1024, 4>(a, s);
        case 4: return a.dim <= kFew4 ? fwd_one<T, TO, kLayer, 4, 512, 4>(a, s) : fwd_one<T, TO, kLayer, 4, 1024, 8>(a, s);
        default: return a.dim <= kFew8 ? fwd_one<T, TO, kLayer, 8, 256, 8>(a, s) : fwd_one<T, TO, kLayer, 8, 1024, 8>(a, s);
    }
}
template <typename T, typename TO>
hipError_t layer_bwd_t(const NormArgs& a, hipStream_t s) {
    hipError_t e;
    const bool f32 = sizeof(T) == 4;
    switch (norm_lanes(a.rows, a.seqlen, f32)) {
        case 1: e = bwd_one<T, TO, kLayer, 1, 1024, 4>(a, s); break;
        case 4: e = a.dim <= kFew4 ? bwd_one<T, TO, kLayer, 4, 512, 4>(a, s) : bwd_one<T, TO, kLayer, 4, 1024, 8>(a, s); break;
        default: e = a.dim <= kFew8 ? bwd_one<T, TO, kLayer, 8, 256, 8>(a, s) : bwd_one<T, TO, kLayer, 8, 1024, 8>(a, s); break;
    }
    if (e) return e;
    hipLaunchKernelGGL(norm_partial_sums, dim3((unsigned)((2 * a.dim + kFinCols - 1) / kFinCols)), dim3(kFinCols * kFinRows), 0, s,
                       a.partial, a.dw, a.db, norm_tiles(a.rows, a.seqlen, f32), a.dim);
    return hipGetLastError();
}

// A head's features are few: all stay in registers up to 256 of them.  Us with 256 threads and 512 (batch x heads x features x
// tokens, bf16; forward, backward): 8 x 16 x 64 x 4096 31, 33 and 47, 40; x 128 44, 61 and 50, 64; x 256 100, 167 and 84, 146.  Rows
// of up to two vectors, one lane of 64 threads a tile and eight: 64 x 16 x 128 x 1 backward 4.5, 10.
template <typename T, typename TO, bool BWD>
hipError_t length_t(const NormArgs& a, hipStream_t s) {
    if (!BWD && a.seqlen == 1) return token_t<T, TO, kLength>(a, s);
    constexpr int PER = Storage<T>::kPerVec, G64 = 64 / PER;
    const auto one = [&](auto lanes, auto threads, auto kept) {
        if constexpr (BWD) return bwd_one<T, TO, kLength, decltype(lanes)::value, decltype(threads)::value, decltype(kept)::value>(a, s);
        else return fwd_one<T, TO, kLength, decltype(lanes)::value, decltype(threads)::value, decltype(kept)::value>(a, s);
    };
    using std::integral_constant;
    if (a.seqlen <= 2 * PER) return one(integral_constant<int, 1>{}, integral_constant<int, 64>{}, integral_constant<int, 4>{});
    if (a.dim <= 128) return one(integral_constant<int, G64>{}, integral_constant<int, 256>{}, integral_constant<int, 32 / PER>{});
    return one(integral_constant<int, G64>{}, integral_constant<int, 512>{}, integral_constant<int, 32 / PER>{});
}

}  // namespace

#define PM_NORM_TYPES(CALL)                                      \
    switch (a.dtype) {                                           \
        case 1: return CALL(bf16_t, bf16_t);                     \
        case 2: return CALL(bf16_t, float);                      \
        default: return CALL(float, float);                      \
    }
#define PM_LAYER_FWD(T, TO) layer_fwd_t<T, TO>(a, s)
#define PM_LAYER_BWD(T, TO) layer_bwd_t<T, TO>(a, s)
#define PM_LENGTH_FWD(T, TO) length_t<T, TO, false>(a, s)
#define PM_LENGTH_BWD(T, TO) length_t<T, TO, true>(a, s)
hipError_t launch_layernorm_fwd(const NormArgs& a, hipStream_t s) { PM_NORM_TYPES(PM_LAYER_FWD) }
hipError_t launch_layernorm_bwd(const NormArgs& a, hipStream_t s) { PM_NORM_TYPES(PM_LAYER_BWD) }
hipError_t launch_l2norm_fwd(const NormArgs& a, hipStream_t s) { PM_NORM_TYPES(PM_LENGTH_FWD) }
hipError_t launch_l2norm_bwd(const NormArgs& a, hipStream_t s) { PM_NORM_TYPES(PM_LENGTH_BWD) }
#undef PM_LENGTH_BWD
#undef PM_LENGTH_FWD
#undef PM_LAYER_BWD
#undef PM_LAYER_FWD
#undef PM_NORM_TYPES

}  // namespace pm
