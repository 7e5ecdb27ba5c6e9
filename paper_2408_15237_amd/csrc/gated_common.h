// What the forward and the backward pass of the gated recurrence share: how lanes lie over channels and tokens, and the loads of a tile.
#pragma once

#include "layers_internal.h"

namespace ssmv {

constexpr int kGatedWaves = 8, kGatedRun = 8;       // waves of a workgroup; tokens that a lane takes one after the other

// A lane owns 4 bytes of a token's row (two bf16 channels, one fp32) for kGatedRun tokens: lane l of a wave the channels l % CL and the run of tokens l / CL.
template <int IO, int CL>
struct GatedLane {
    static constexpr int CH = IO == SSMV_BF16 ? 2 : 1, ES = IO == SSMV_BF16 ? 2 : 4;
    static constexpr int G = 64 / CL, T = kGatedWaves * G * kGatedRun;      // runs of a wave; tokens of a tile
    static constexpr int CW = CL * CH;                                      // channels of a workgroup

    static __device__ __forceinline__ void decode(uint32_t w, float (&v)[CH])
    {
        if constexpr (IO == SSMV_BF16) {
            v[0] = __uint_as_float(w << 16);
            v[1] = __uint_as_float(w & 0xffff0000u);
        } else {
            v[0] = __uint_as_float(w);
        }
    }
    static __device__ __forceinline__ uint32_t load(const char *row, unsigned off, int live)
    {
        uint32_t r = 0;
        if (live == CH) __builtin_memcpy(&r, row + off, 4);
        else if (live > 0) r = *reinterpret_cast<const uint16_t *>(row + off);
        return r;
    }
    static __device__ __forceinline__ void store(char *row, unsigned off, int live, const float (&v)[CH])
    {
        if (live == CH) {
            uint32_t r;
            if constexpr (IO == SSMV_BF16) r = pack_bf16x2(v[0], v[CH - 1]);
            else r = __float_as_uint(v[0]);
            __builtin_memcpy(row + off, &r, 4);
        } else if (live > 0) {
            *reinterpret_cast<uint16_t *>(row + off) = f32_to_bf16_bits(v[0]);
        }
    }
    // the run's tokens from t on, of `len`: what is behind them counts as zeros and is not read
    static __device__ __forceinline__ void load_run(uint32_t (&r)[kGatedRun], const void *base, size_t stride, size_t wave_token, unsigned off, int live, int t, int len)
    {
        const char *row = static_cast<const char *>(base) + wave_token * stride * ES;
#pragma unroll
        for (int k = 0; k < kGatedRun; ++k) {
            r[k] = 0;
            if (t + k < len) r[k] = load(row + k * stride * ES, off, live);
        }
    }
};

// CH floats of a row of states or of a vector
template <int CH>
__device__ __forceinline__ void load_channels(const float *from, int live, float (&v)[CH], float missing = 0.f)
{
#pragma unroll
    for (int c = 0; c < CH; ++c) v[c] = c < live ? from[c] : missing;
}
template <int CH>
__device__ __forceinline__ void store_channels(float *to, int live, const float (&v)[CH])
{
#pragma unroll
    for (int c = 0; c < CH; ++c)
        if (c < live) to[c] = v[c];
}

}  // namespace ssmv
