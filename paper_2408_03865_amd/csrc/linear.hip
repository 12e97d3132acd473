// linear.hip -- linear attention beside the walks (linear_walk.hpp): which kernel a walk takes, the
// states of split rows, the decay's gradient and the sums over the heads that share q and k.
#include "linear_walk.hpp"

namespace pm {

extern template hipError_t launch_walk_kc<float, float, 64>(const WalkArgs&, WalkMode, bool, hipStream_t);
extern template hipError_t launch_walk_kc<float, float, 128>(const WalkArgs&, WalkMode, bool, hipStream_t);
extern template hipError_t launch_walk_kc<bf16_t, bf16_t, 64>(const WalkArgs&, WalkMode, bool, hipStream_t);
extern template hipError_t launch_walk_kc<bf16_t, bf16_t, 128>(const WalkArgs&, WalkMode, bool, hipStream_t);
extern template hipError_t launch_walk_kc<bf16_t, float, 64>(const WalkArgs&, WalkMode, bool, hipStream_t);
extern template hipError_t launch_walk_kc<bf16_t, float, 128>(const WalkArgs&, WalkMode, bool, hipStream_t);

namespace {

template <typename T, typename TO>
hipError_t walk_t(const WalkArgs& a, WalkMode mode, bool exact, hipStream_t s) {
    return a.x.rows <= 64 ? launch_walk_kc<T, TO, 64>(a, mode, exact, s) : launch_walk_kc<T, TO, 128>(a, mode, exact, s);
}

// The state that enters each segment, in place of what the segment before it in the walk adds:
// cur <- A cur + added, one thread an element.  Bound by latency: 4 x 24 heads x 5 segments of 64 x 64 take 5.5 us.
__global__ void walk_chain(float* __restrict__ seg, const float* __restrict__ seg_a, const float* __restrict__ entry,
                           int64_t sz, int nseg, int rev) {
    const int64_t parts = (sz + blockDim.x - 1) / blockDim.x, bh = blockIdx.x / parts;
    const int64_t i = (blockIdx.x - bh * parts) * blockDim.x + threadIdx.x;
    if (i >= sz) return;
    float cur = entry ? entry[bh * sz + i] : 0.0f;
    const int64_t step = rev ? -sz : sz;
    float* p = seg + (bh * nseg + (rev ? nseg - 1 : 0)) * sz + i;
    const float* pa = seg_a + bh * nseg + (rev ? nseg - 1 : 0);
    // the last segment adds to nothing; eight loads on their way at a time
    for (int k = 0; k < nseg; k += 8) {
        float added[8], A[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (k + j + 1 < nseg) {
                added[j] = p[(k + j) * step];
                A[j] = pa[rev ? -(k + j) : k + j];
            }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (k + j >= nseg) break;
            p[(k + j) * step] = cur;
            if (k + j + 1 < nseg) cur = A[j] < 0.0f ? added[j] : fmaf(A[j], cur, added[j]);
        }
    }
}

template <typename T, int KC, int VP>
hipError_t aggregate_vp(const WalkArgs& a, hipStream_t s) {
    constexpr int NS = Mat<T>::kSplit ? 3 : 1;
    const dim3 grid((unsigned)((int64_t)a.batch * a.heads * (a.nseg - 1))), block(walk_threads(VP, walk_parts<T, KC, VP>()));
    if (a.rev) hipLaunchKernelGGL((walk_aggregate<T, KC, VP, true, NS>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((walk_aggregate<T, KC, VP, false, NS>), grid, block, 0, s, a);
    return hipGetLastError();
}

template <typename T, int KC>
hipError_t aggregate_kc(const WalkArgs& a, hipStream_t s) {
    return a.z.rows <= 64 ? aggregate_vp<T, KC, 64>(a, s) : aggregate_vp<T, KC, 128>(a, s);
}

template <typename T>
hipError_t aggregate_t(const WalkArgs& a, hipStream_t s) {
    return a.x.rows <= 64 ? aggregate_kc<T, 64>(a, s) : aggregate_kc<T, 128>(a, s);
}

// ddecay at t: the sum of r = rq + rk over t and the tokens after it in its sequence up to the next
// boundary, plus the product of the two states there if the sequence goes on.  One wave a piece of
// a row between two boundaries, from its end in steps of 64 tokens.  8 x 32 rows of 4096 tokens: 14 us, 1.5% of the backward.
__global__ __launch_bounds__(256) void linear_ddecay_kernel(LinDecayArgs a) {
    const int64_t id = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 6;
    const int l = lane_id();
    const int64_t bh = id / a.nb;
    if (bh >= (int64_t)a.batch * a.heads) return;
    const int n = (int)(id - bh * a.nb);
    const int64_t b = bh / a.heads, h = bh - b * a.heads, L = a.seqlen;
    const int64_t t0 = (int64_t)n * a.bound_tokens, t1 = min(L, t0 + a.bound_tokens);
    const int32_t* pos = a.pos + b * L;
    const float* rq = a.rq + bh * L;
    const float* rk = a.rk + bh * L;
    const auto cut = [&](int64_t t) {
        const float g = a.decay_mode == 2 ? a.decay[bh * L + t] : a.decay[h];
        return pos[t] == 0 || g <= kDecayCut;
    };
    // what lies past the boundary
    float carry = 0.0f;
    if (t1 < L ? !cut(t1) : a.bound_end != 0) carry = a.dot[bh * (a.nb + 1) + n + 1];
    float sum = 0.0f;
    for (int64_t e = t1; e > t0; e -= 64) {          // lane l: token e - 1 - l
        const int64_t t = e - 1 - l;
        const bool in = t >= t0;
        float v = in ? rq[t] + rk[t] : 0.0f;
        const bool c = in && cut(t);
        // sums over the lanes before (the tokens after): a start's own r is in, nothing passes it
        const int start = c ? 1 : 0;
        float acc = v;
        int f = __shfl_up(start, 1);             // a start among the lanes summed, this lane's left out
        if (l == 0) f = 0;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const float pv = __shfl_up(acc, m);
            const int pf = __shfl_up(f, m);
            if (l >= m && !f) {
                acc += pv;
                f = pf;
            }
        }
        const float dg = f ? acc : acc + carry;
        const float res = c ? 0.0f : dg;
        if (in && a.decay_mode == 2) a.ddecay[bh * L + t] = res;
        if (in) sum += res;
        // to the tokens before: nothing if the step's first token starts a sequence
        const float lastv = __shfl(dg, 63);
        const int lastc = __shfl(start, 63);
        carry = lastc ? 0.0f : lastv;
    }
    if (a.decay_mode == 1) {
#pragma unroll
        for (int m = 1; m < 64; m *= 2) sum += __shfl_xor(sum, m);
        if (l == 0) a.partial[(h * a.batch + b) * a.nb + n] = sum;
    }
}

// ddecay[h] from its pieces, one wave a head, in a fixed order
__global__ __launch_bounds__(64) void linear_ddecay_heads(const float* __restrict__ partial, float* __restrict__ ddecay,
                                                          int64_t n) {
    float v = 0.0f;
    for (int64_t i = threadIdx.x; i < n; i += 64) v += partial[blockIdx.x * n + i];
#pragma unroll
    for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
    if (threadIdx.x == 0) ddecay[blockIdx.x] = v;
}

// The sum over the heads of a group, in their order: four elements a thread, 1024 a block of one (batch, group).  Bound by
// the 32-bit parts it reads: 8 x 32 heads of 128 x 4096, groups of 4, 604 MB in 89 us, 6.8 TB/s (some from the last
// cache); 2 x 24 heads of 64 x 512, one group, 3.8 us, with one load at a time 8.7.
constexpr int kSumAhead = 8;            // heads' loads on their way at a time
template <typename TO>
__global__ __launch_bounds__(256) void group_sum_kernel(const float* __restrict__ part, TO* __restrict__ out, int per, int64_t n,
                                                        const float* __restrict__ part1, TO* __restrict__ out1) {
    if (blockIdx.y) {
        part = part1;
        out = out1;
    }
    const int64_t blocks = (n + 1023) / 1024, bg = blockIdx.x / blocks;
    const int64_t i = (blockIdx.x - bg * blocks) * 1024 + threadIdx.x * 4;
    if (i >= n) return;
    const float* p = part + bg * per * n + i;
    TO* o = out + bg * n + i;
    if (i + 4 <= n) {
        f32x4 v = {0, 0, 0, 0};
        int k = 0;
        for (; k + kSumAhead <= per; k += kSumAhead) {
            f32x4 w[kSumAhead];
#pragma unroll
            for (int j = 0; j < kSumAhead; ++j) w[j] = __builtin_bit_cast(f32x4, u32x4(load_vec<float, 4, true>(p + (k + j) * n)));
#pragma unroll
            for (int j = 0; j < kSumAhead; ++j) v += w[j];
        }
        for (; k < per; ++k) v += __builtin_bit_cast(f32x4, u32x4(load_vec<float, 4, true>(p + k * n)));
        if constexpr (sizeof(TO) == 2) *reinterpret_cast<u32x2_a2*>(o) = Mat<bf16_t>::round(v);
        else *reinterpret_cast<u32x4_a4*>(o) = __builtin_bit_cast(u32x4, v);
    } else {
        for (int r = 0; i + r < n; ++r) {
            float v = p[r];
            for (int k = 1; k < per; ++k) v += p[k * n + r];
            Storage<TO>::store1(o + r, v);
        }
    }
}

// of one tensor, or of two in one launch
hipError_t group_sums(const float* part, void* out, const float* part1, void* out1, int64_t batch, int32_t heads, int32_t groups,
                      int64_t n, bool f32, hipStream_t s) {
    const dim3 grid((unsigned)((n + 1023) / 1024 * batch * groups), part1 ? 2 : 1);
    if (f32)
        hipLaunchKernelGGL(group_sum_kernel<float>, grid, dim3(256), 0, s, part, static_cast<float*>(out), heads / groups, n, part1,
                           static_cast<float*>(out1));
    else
        hipLaunchKernelGGL(group_sum_kernel<bf16_t>, grid, dim3(256), 0, s, part, static_cast<bf16_t*>(out), heads / groups, n, part1,
                           static_cast<bf16_t*>(out1));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_walk(const WalkArgs& a, WalkMode mode, bool exact, hipStream_t s) {
    switch (a.dtype) {
        case 1: return walk_t<bf16_t, bf16_t>(a, mode, exact, s);
        case 2: return walk_t<bf16_t, float>(a, mode, exact, s);
        default: return walk_t<float, float>(a, mode, exact, s);
    }
}

hipError_t launch_walk_segments(const WalkArgs& a, hipStream_t s) {
    if (hipError_t e = a.dtype == 0 ? aggregate_t<float>(a, s) : aggregate_t<bf16_t>(a, s)) return e;
    const int64_t sz = (int64_t)a.x.rows * a.z.rows;
    hipLaunchKernelGGL(walk_chain, dim3((unsigned)((sz + 255) / 256 * a.batch * a.heads)), dim3(256), 0, s,
                       a.seg, a.seg_a, a.entry, sz, a.nseg, a.rev);
    return hipGetLastError();
}

hipError_t launch_linear_ddecay(const LinDecayArgs& a, hipStream_t s) {
    const int64_t waves = (int64_t)a.batch * a.heads * a.nb;
    hipLaunchKernelGGL(linear_ddecay_kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
    if (a.decay_mode != 1) return hipSuccess;
    hipLaunchKernelGGL(linear_ddecay_heads, dim3((unsigned)a.heads), dim3(64), 0, s, a.partial, a.ddecay,
                       (int64_t)a.batch * a.nb);
    return hipGetLastError();
}

hipError_t launch_linear_group_sum(const float* part, void* out, int64_t batch, int32_t heads, int32_t groups, int64_t n,
                                   bool f32, hipStream_t s) {
    return group_sums(part, out, nullptr, nullptr, batch, heads, groups, n, f32, s);
}

hipError_t launch_linear_group_sums(const float* part, void* out, const float* part1, void* out1, int64_t batch, int32_t heads,
                                    int32_t groups, int64_t n, bool f32, hipStream_t s) {
    return group_sums(part, out, part1, out1, batch, heads, groups, n, f32, s);
}

}  // namespace pm
