// linear_step.hip -- linear attention of one token a sequence: S <- a S + k v^T, out = scale S^T q, the
// state (dk, dv) of every batch row and head read and written in place, in 32 bits.
// Bound by the state's bytes, 8 dk dv a head.  A block takes one head of one batch row, or some of its
// columns where heads are few: LPR lanes of four consecutive columns side by side, 256 / LPR rows at once, all of a
// thread's rows loaded before the first is used.
#include "common.hpp"
#include "linear.hpp"

namespace pm {
namespace {

typedef f32x4 f32x4_a4 __attribute__((aligned(4)));
constexpr int kThreads = 256;
constexpr float kStepCut = -104.0f;      // as a chunk's decays: exp of it is 0 in 32 bits

template <bool ALIGNED>
__device__ __forceinline__ f32x4 load4(const float* p) {
    if constexpr (ALIGNED) return *reinterpret_cast<const f32x4*>(p);
    else return *reinterpret_cast<const f32x4_a4*>(p);
}
template <bool ALIGNED>
__device__ __forceinline__ void store4(float* p, const f32x4& v) {
    if constexpr (ALIGNED) *reinterpret_cast<f32x4*>(p) = v;
    else *reinterpret_cast<f32x4_a4*>(p) = v;
}

// WHOLE: a row of the state is whole vectors, 16-byte aligned; else vectors have an element's alignment and a row's
// last columns go one by one.
template <typename T, typename TO, bool WHOLE, int LPR>
__global__ __launch_bounds__(kThreads) void step_kernel(LinStepArgs a) {
    constexpr int VEC = 4, R = kThreads / LPR, kCols = LPR * VEC, kAhead = R >= 16 ? 8 : 16;
    __shared__ float qk[2][kLinMaxHead];
    __shared__ float red[kThreads / 64][kCols];
    const int parts = (a.dv + kCols - 1) / kCols;
    const int64_t bh = blockIdx.x / parts;
    const int part = (int)(blockIdx.x - bh * parts);
    const int64_t b = bh / a.heads, h = bh - b * a.heads;
    const int lane = threadIdx.x % LPR, row = threadIdx.x / LPR;
    const int c = part * kCols + lane * VEC;
    const bool live = c < a.dv, vector = WHOLE ? live : c + VEC <= a.dv;
    const int p = a.pos ? a.pos[b] : 1;
    TO* out = static_cast<TO*>(a.out) + bh * a.dv;
    if (p < 0) {                                          // an idle row
        if (row == 0 && live) {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (WHOLE || c + i < a.dv) Storage<TO>::store1(out + c + i, 0.0f);
        }
        return;
    }
    const float g = a.decay_mode == 2 ? a.decay[bh] : a.decay_mode == 1 ? a.decay[h] : 0.0f;
    const bool cut = p == 0 || g <= kStepCut;
    const float decay = expf(g);
    float* st = a.state + (bh * a.dk) * (int64_t)a.dv + c;
    const int64_t gq = (b * a.groups + h / (a.heads / a.groups)) * a.dk;
    const T* q = static_cast<const T*>(a.q) + gq;
    const T* k = static_cast<const T*>(a.k) + gq;
    float v[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = c + i < a.dv ? Storage<T>::load1(static_cast<const T*>(a.v) + bh * a.dv + c + i) : 0.0f;
    float acc[VEC] = {};
    bool staged = false;
    for (int f0 = 0; f0 < a.dk; f0 += R * kAhead) {
        float s[kAhead][VEC];
#pragma unroll
        for (int n = 0; n < kAhead; ++n) {
            const int f = f0 + n * R + row;
#pragma unroll
            for (int i = 0; i < VEC; ++i) s[n][i] = 0.0f;
            if (f < a.dk && vector && !cut) {
                const f32x4 w = load4<WHOLE>(st + f * a.dv);
#pragma unroll
                for (int i = 0; i < VEC; ++i) s[n][i] = w[i];
            }
            if (!WHOLE && f < a.dk && live && !vector && !cut) {
#pragma unroll
                for (int i = 0; i < VEC - 1; ++i)
                    if (c + i < a.dv) s[n][i] = st[f * a.dv + i];
            }
        }
        if (!staged) {                                    // block-uniform
            if (threadIdx.x < 2 * kLinMaxHead) {
                const int f = threadIdx.x % kLinMaxHead;
                if (f < a.dk) qk[threadIdx.x / kLinMaxHead][f] = Storage<T>::load1((threadIdx.x < kLinMaxHead ? q : k) + f);
            }
            __syncthreads();
            staged = true;
        }
#pragma unroll
        for (int n = 0; n < kAhead; ++n) {
            const int f = f0 + n * R + row;
            if (f < a.dk && live) {
                const float qf = qk[0][f], kf = qk[1][f];
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    s[n][i] = cut ? kf * v[i] : fmaf(decay, s[n][i], kf * v[i]);
                    acc[i] = fmaf(qf, s[n][i], acc[i]);
                }
                if (vector) {
                    store4<WHOLE>(st + f * a.dv, f32x4{s[n][0], s[n][1], s[n][2], s[n][3]});
                } else if (!WHOLE) {
#pragma unroll
                    for (int i = 0; i < VEC - 1; ++i)
                        if (c + i < a.dv) st[f * a.dv + i] = s[n][i];
                }
            }
        }
    }
#pragma unroll
    for (int m = LPR; m < 64; m *= 2)
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] += __shfl_xor(acc[i], m);
    if ((threadIdx.x & 63) < LPR) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) red[threadIdx.x >> 6][lane * VEC + i] = acc[i];
    }
    __syncthreads();
    if (threadIdx.x < kCols && part * kCols + (int)threadIdx.x < a.dv) {
        float o = red[0][threadIdx.x];
#pragma unroll
        for (int w = 1; w < kThreads / 64; ++w) o += red[w][threadIdx.x];
        Storage<TO>::store1(out + part * kCols + threadIdx.x, o * a.scale);
    }
}

template <typename T, typename TO, bool WHOLE, int LPR>
hipError_t step_one(const LinStepArgs& a, hipStream_t s) {
    const int64_t parts = (a.dv + LPR * 4 - 1) / (LPR * 4);
    hipLaunchKernelGGL((step_kernel<T, TO, WHOLE, LPR>), dim3((unsigned)((int64_t)a.batch * a.heads * parts)), dim3(kThreads),
                       0, s, a);
    return hipGetLastError();
}

// 64 columns of the state in 16-byte vectors, or 16 where the heads alone leave most CUs idle.  Us with 16 and 64 (heads,
// dk x dv): 24, 64 x 64 4.2, 4.5; 24, 128 x 64 4.5, 5.3; 96, 64 x 64 5.1, 4.7; 160, 128 x 64 7.7, 5.9; 1024, 128 x 128
// 38, 24 (all 128 columns 25).  4096 heads of 128 x 64 take 57 us, 4.7 TB/s of states read and written, a large
// copy's rate.
template <typename T, typename TO, bool WHOLE>
hipError_t step_w(const LinStepArgs& a, hipStream_t s) {
    return (int64_t)a.batch * a.heads <= 64 ? step_one<T, TO, WHOLE, 4>(a, s) : step_one<T, TO, WHOLE, 16>(a, s);
}
template <typename T, typename TO>
hipError_t step_t(const LinStepArgs& a, hipStream_t s) {
    return a.dv % 4 ? step_w<T, TO, false>(a, s) : step_w<T, TO, true>(a, s);
}

}  // namespace

hipError_t launch_linear_step(const LinStepArgs& a, hipStream_t s) {
    switch (a.dtype) {
        case 1: return step_t<bf16_t, bf16_t>(a, s);
        case 2: return step_t<bf16_t, float>(a, s);
        default: return step_t<float, float>(a, s);
    }
}

}  // namespace pm
