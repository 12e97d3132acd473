// norms.hpp -- host-side launchers of the layer norm and of the norm by a head's length (norms.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace pm {

// (rows, dim, seqlen): the layer norm's rows are those of the batch, the other's those of the batch's groups.
struct NormArgs {
    const void* x;
    const void* dout;           // backward
    const void* dres;           // backward: added to dx, or null
    const float* w;             // layer norm
    const float* b;             // layer norm, or null
    const float* mean;          // backward, layer norm
    const float* rstd;          // backward
    void* out;                  // out, or dx
    float* mean_out;
    float* rstd_out;
    float* partial;             // layer norm backward: (tiles, 2, dim)
    float* dw;
    float* db;
    float eps;
    int64_t rows, dim, seqlen;
    int32_t dtype;              // 0 fp32, 1 bf16, 2 bf16 with fp32 out
};

// Tokens of a block's tile: LANES vectors of 16 bytes, so that every feature's row gives LANES x 16 consecutive bytes.
// 128 of them are whole lines; fewer where that leaves CUs without a tile, in fp32, whose tile has half the tokens, from
// 128 tiles on.  Us with 64 and 128 bytes (batch x features x tokens, layer norm's forward, backward; bf16 but the last):
//   8 x 2048 x 4096 (512 tiles of 128) 82, 72; 169, 144    4 x 8192 x 2048 (128) 82, 104; 205, 248    2 x 2560 x 3001 (94) 44, 48; 68, 99
//   8 x 768 x 4096 41, 29; 74, 56                          fp32 2 x 2560 x 3001 (188) 68, 52; 105, 89
inline int norm_lanes(int64_t rows, int64_t seqlen, bool f32) {
    const int64_t per = f32 ? 4 : 8;
    const auto tiles = [&](int lanes) { return rows * ((seqlen + lanes * per - 1) / (lanes * per)); };
    if (seqlen <= per || tiles(4) < 128) return 1;
    return tiles(8) < (f32 ? 128 : 256) ? 4 : 8;
}
inline int64_t norm_tiles(int64_t rows, int64_t seqlen, bool f32) {
    const int64_t tile = (int64_t)norm_lanes(rows, seqlen, f32) * (f32 ? 4 : 8);
    return rows * ((seqlen + tile - 1) / tile);
}

hipError_t launch_layernorm_fwd(const NormArgs& a, hipStream_t s);
hipError_t launch_layernorm_bwd(const NormArgs& a, hipStream_t s);
hipError_t launch_l2norm_fwd(const NormArgs& a, hipStream_t s);
hipError_t launch_l2norm_bwd(const NormArgs& a, hipStream_t s);

}  // namespace pm
