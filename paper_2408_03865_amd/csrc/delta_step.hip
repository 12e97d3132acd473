// delta_step.hip -- the gated delta rule for one token a sequence, in 32 bits: with S' = a S,
//   u = beta (v - S'^T k),  S <- S' + k u^T,  out = scale S^T q = scale (S'^T q + (k . q) u),
// the state (dk, dv) of every batch row and head read and written in place.
// Bound by the state's bytes, 8 dk dv a head.  A block takes 64 columns of one head of one batch row: 16 lanes of four consecutive
// ones side by side, 16 rows at once.  All of a thread's rows, eight at most, stay in registers between the two products with the
// state, which are summed over the rows together, and its update; 96 registers a thread leave room for five blocks a CU (64 x 32
// heads of 128 x 128: 59 us, 4.6 TB/s of states read and written; with the 203 that the compiler takes by itself 92).
#include "common.hpp"
#include "delta.hpp"

namespace pm {
namespace {

typedef f32x4 f32x4_a4 __attribute__((aligned(4)));
// Lanes beside each other: with four, 24 heads of 64 x 64 take 3.9 us and not 4.1, 64 of 128 x 128 6.6 and not 4.8.
constexpr int kThreads = 256, LPR = 16;
constexpr float kStepCut = -104.0f;      // as a chunk's decays: exp of it is 0 in 32 bits

// WHOLE: a row of the state is whole vectors, 16-byte aligned; else vectors have an element's alignment and a row's
// last columns go one by one.
template <typename T, typename TO, bool WHOLE>
__global__ __launch_bounds__(kThreads, 5) void delta_step_kernel(DeltaStepArgs a) {
    constexpr int VEC = 4, R = kThreads / LPR, kCols = LPR * VEC, kRows = (kLinMaxHead + R - 1) / R, kWaves = kThreads / 64;
    __shared__ float qk[2][kLinMaxHead];
    __shared__ float red[2][kWaves][kCols];
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
    const float decay = expf(g), beta = a.beta[bh];
    float* st = a.state + (bh * a.dk) * (int64_t)a.dv + c;
    const int64_t gq = (b * a.groups + h / (a.heads / a.groups)) * a.dk;
    f32x4 s[kRows];
#pragma unroll
    for (int n = 0; n < kRows; ++n) {
        const int f = n * R + row;
        s[n] = f32x4{0, 0, 0, 0};
        if (f >= a.dk || cut) continue;
        if (vector) {
            if constexpr (WHOLE) s[n] = *reinterpret_cast<const f32x4*>(st + f * a.dv);
            else s[n] = *reinterpret_cast<const f32x4_a4*>(st + f * a.dv);
        } else if (!WHOLE && live) {
#pragma unroll
            for (int i = 0; i < VEC - 1; ++i)
                if (c + i < a.dv) s[n][i] = st[f * a.dv + i];
        }
    }
    f32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < VEC; ++i)
        if (c + i < a.dv) v[i] = Storage<T>::load1(static_cast<const T*>(a.v) + bh * a.dv + c + i);
    {
        const int f = threadIdx.x % kLinMaxHead;
        const T* from = static_cast<const T*>(threadIdx.x < kLinMaxHead ? a.q : a.k) + gq;
        qk[threadIdx.x / kLinMaxHead][f] = f < a.dk ? Storage<T>::load1(from + f) : 0.0f;
    }
    __syncthreads();
    const int l = threadIdx.x & 63;
    float dot = fmaf(qk[0][l], qk[1][l], qk[0][l + 64] * qk[1][l + 64]);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) dot += __shfl_xor(dot, m);
    f32x4 sk = {0, 0, 0, 0}, sq = {0, 0, 0, 0};
#pragma unroll
    for (int n = 0; n < kRows; ++n) {
        const int f = min(n * R + row, kLinMaxHead - 1);
        if (!cut) s[n] *= decay;
        sk += s[n] * qk[1][f];
        sq += s[n] * qk[0][f];
    }
#pragma unroll
    for (int m = LPR; m < 64; m *= 2)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            sk[i] += __shfl_xor(sk[i], m);
            sq[i] += __shfl_xor(sq[i], m);
        }
    if (l < LPR) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            red[0][threadIdx.x >> 6][lane * VEC + i] = sk[i];
            red[1][threadIdx.x >> 6][lane * VEC + i] = sq[i];
        }
    }
    __syncthreads();
    f32x4 u, o;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        float k1 = red[0][0][lane * VEC + i], q1 = red[1][0][lane * VEC + i];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
            k1 += red[0][w][lane * VEC + i];
            q1 += red[1][w][lane * VEC + i];
        }
        u[i] = beta * (v[i] - k1);
        o[i] = a.scale * fmaf(dot, u[i], q1);
    }
    if (!live) return;
    if (row == 0) {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (WHOLE || c + i < a.dv) Storage<TO>::store1(out + c + i, o[i]);
    }
#pragma unroll
    for (int n = 0; n < kRows; ++n) {
        const int f = n * R + row;
        if (f >= a.dk) continue;
        s[n] += qk[1][f] * u;
        if (vector) {
            if constexpr (WHOLE) *reinterpret_cast<f32x4*>(st + f * a.dv) = s[n];
            else *reinterpret_cast<f32x4_a4*>(st + f * a.dv) = s[n];
        } else if (!WHOLE) {
#pragma unroll
            for (int i = 0; i < VEC - 1; ++i)
                if (c + i < a.dv) st[f * a.dv + i] = s[n][i];
        }
    }
}

template <typename T, typename TO, bool WHOLE>
hipError_t step_w(const DeltaStepArgs& a, hipStream_t s) {
    const int64_t parts = (a.dv + LPR * 4 - 1) / (LPR * 4);
    hipLaunchKernelGGL((delta_step_kernel<T, TO, WHOLE>), dim3((unsigned)((int64_t)a.batch * a.heads * parts)), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}
template <typename T, typename TO>
hipError_t step_t(const DeltaStepArgs& a, hipStream_t s) {
    return a.dv % 4 ? step_w<T, TO, false>(a, s) : step_w<T, TO, true>(a, s);
}

}  // namespace

hipError_t launch_delta_step(const DeltaStepArgs& a, hipStream_t s) {
    switch (a.dtype) {
        case 1: return step_t<bf16_t, bf16_t>(a, s);
        case 2: return step_t<bf16_t, float>(a, s);
        default: return step_t<float, float>(a, s);
    }
}

}  // namespace pm
