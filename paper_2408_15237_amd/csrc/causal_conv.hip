// The causal depthwise convolution of width 4 from a history of raw inputs to the newest one, over a prompt or one token of every row,
// and the conv part of a cache's state.
#include "decode_internal.h"

namespace ssmv {
namespace {

constexpr int W = SSMV_CONV_WIDTH;

// VEC elements of one token row: 16 bytes, at the alignment of an element (aligned ones are as fast, others still much faster than an
// element at a time), or one element where a row has fewer
template <int IO, int VEC>
struct Chunk {
    using Vec = IoVec<IO>;
    static constexpr int ES = IO == SSMV_BF16 ? 2 : 4;
    static __device__ __forceinline__ uint4 zero() { return make_uint4(0, 0, 0, 0); }
    static __device__ __forceinline__ uint4 load(const void *base, size_t idx)
    {
        if constexpr (VEC > 1) {
            uint4 r;
            __builtin_memcpy(&r, static_cast<const char *>(base) + idx * ES, sizeof(r));
            return r;
        } else {
            return make_uint4(Vec::load_raw1(base, idx), 0, 0, 0);
        }
    }
    // its elements from `skip` on; PAST: past the caches
    template <bool PAST>
    static __device__ __forceinline__ void store(void *base, size_t idx, uint4 r, int skip)
    {
        if constexpr (VEC == 1) {
            Vec::store_raw1(base, idx, r.x);
        } else if (skip == 0) {
            typedef uint32_t loose __attribute__((ext_vector_type(4), aligned(2)));
            loose *to = reinterpret_cast<loose *>(static_cast<char *>(base) + idx * ES);
            const loose v = {r.x, r.y, r.z, r.w};
            if constexpr (PAST) __builtin_nontemporal_store(v, to);
            else *to = v;
        } else {
            const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int j = 1; j < VEC; ++j)
                if (j >= skip) Vec::store_raw1(base, idx + j, IO == SSMV_BF16 ? w[j / 2] >> (j % 2 * 16) : w[j % 4]);
        }
    }
    static __device__ __forceinline__ void decode(uint4 r, float (&v)[VEC])
    {
        if constexpr (VEC > 1) Vec::decode(r, v);
        else v[0] = Vec::decode1(r.x);
    }
    static __device__ __forceinline__ uint4 encode(const float (&v)[VEC])
    {
        if constexpr (VEC > 1) return Vec::encode(v);
        else if constexpr (IO == SSMV_BF16) return make_uint4(f32_to_bf16_bits(v[0]), 0, 0, 0);
        else return make_uint4(__float_as_uint(v[0]), 0, 0, 0);
    }
};

// Bound by memory: a token row in, a token row out (8 x 2048 x 5120 bf16, 336 MB, other tensors in every call: 60.5 to 62.6 us, 5.4 to 5.5 TB/s; copies of 1 GB 5.1 to 6.1).
// A thread owns VEC adjacent channels of T tokens: it requests its tokens and the three before them together, and slides over
// them in registers.  The three are those of the thread of the tokens before, 2^lanes threads ahead in the same workgroup, and come out of the
// L1 - but for the workgroup's first tile, one in 256 / 2^lanes: with 64 vectors side by side one in four, so that 19 tokens are read from beyond
// it for 16 written (8 x 2048 x 5120 bf16: FETCH_SIZE x 2 = 1.19 WRITE_SIZE).  What a workgroup reads does not depend on where others run.  The first tokens
// take the history, and their thread also leaves the newest three inputs, so that conv_out may be conv_in.  (The choice of a history vector by the
// sequence's length, at the end, keeps the three in 64 bytes of scratch memory a lane.)
template <int IO, int VEC, int T, bool PAST>
__global__ __launch_bounds__(256) void causal_conv_kernel(const CausalConvParams p, int lanes, unsigned chunks, unsigned groups)
{
    using Ch = Chunk<IO, VEC>;
    const unsigned b = blockIdx.y, run = blockIdx.x / groups, group = blockIdx.x - run * groups;       // groups of channels; runs of tiles
    const unsigned chunk = (group << lanes) + (threadIdx.x & ((1u << lanes) - 1)), tile = (run << (8 - lanes)) + (threadIdx.x >> lanes);
    if (chunk >= chunks) return;
    // the last channels of a row: moved back to a whole vector, of which only what is the thread's own is stored
    const unsigned c_own = chunk * VEC, c0 = min(c_own, (unsigned)p.C - VEC);
    const int skip = (int)(c_own - c0);
    const int len = p.seq_len ? min(max(p.seq_len[b], 0), p.L) : p.L;
    if (tile * (size_t)T >= (size_t)len && tile != 0) return;
    const int t0 = (int)tile * T;
    const bool first = t0 == 0;

    const size_t row0 = (size_t)b * p.L;                       // the sequence's tokens
    auto x_at = [&](int t) { return Ch::load(p.x, (row0 + t) * p.x_stride + c0); };
    uint4 raw[W - 1 + T];
    uint4 hist[W - 1];
    if (first) {
        const int src = p.src_row ? p.src_row[b] : (int)b;
        const bool have = p.conv_in && (unsigned)src < (unsigned)p.rows_in;
#pragma unroll
        for (int i = 0; i < W - 1; ++i) hist[i] = have ? Ch::load(p.conv_in, ((size_t)src * (W - 1) + i) * p.C + c0) : Ch::zero();
#pragma unroll
        for (int i = 0; i < W - 1; ++i) raw[i] = hist[i];
    } else {
#pragma unroll
        for (int i = 0; i < W - 1; ++i) raw[i] = x_at(t0 - (W - 1) + i);
    }
    if (len > 0) {
        // tokens behind the last one: the last one again, dropped below
#pragma unroll
        for (int i = 0; i < T; ++i) raw[W - 1 + i] = x_at(min(t0 + i, len - 1));
        float w[VEC][W], bias[VEC], v[W][VEC];
        if constexpr (VEC > 1) {
#pragma unroll
            for (int i = 0; i < W; ++i) {                      // 4 VEC adjacent weights: W vectors
                float t[VEC];
                Ch::decode(Ch::load(p.wgt, (size_t)c0 * W + i * VEC), t);
#pragma unroll
                for (int j = 0; j < VEC; ++j) w[(i * VEC + j) / W][(i * VEC + j) % W] = t[j];
            }
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) w[0][i] = load_io(p.wgt, (size_t)c0 * W + i, IO);
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) bias[j] = 0.f;
        if (p.bias) Ch::decode(Ch::load(p.bias, c0), bias);
#pragma unroll
        for (int i = 0; i < W - 1; ++i) Ch::decode(raw[i], v[i]);
#pragma unroll
        for (int i = 0; i < T; ++i) {
            Ch::decode(raw[W - 1 + i], v[(W - 1 + i) % W]);
            if (t0 + i < len) {
                float o[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    o[j] = bias[j];
#pragma unroll
                    for (int k = 0; k < W; ++k) o[j] = fmaf(w[j][k], v[(i + k) % W][j], o[j]);
                    if (p.act == SSMV_ACT_SILU) o[j] = silu_fast(o[j]);
                }
                Ch::template store<PAST>(p.out, (row0 + t0 + i) * p.out_stride + c0, Ch::encode(o), skip);
            }
        }
    }
    if (first && p.conv_out) {
#pragma unroll
        for (int i = 0; i < W - 1; ++i) {
            const int t = len - (W - 1) + i;
            uint4 r;
            if (t >= 0) r = x_at(t);
            else r = len == 0 ? hist[i] : len == 1 ? hist[i + 1 < W - 1 ? i + 1 : i] : hist[W - 2];       // len + i of the history
            Ch::template store<false>(p.conv_out, ((size_t)b * (W - 1) + i) * p.C + c0, r, skip);
        }
    }
}

template <int IO, int VEC>
int launch(const CausalConvParams &p, hipStream_t stream)
{
    const unsigned chunks = (unsigned)((p.C + VEC - 1) / VEC);
    auto go = [&](auto kernel, int T) {
        int lanes = 3;                                                            // up to 64 vectors of a row, the rest of the workgroup the tokens behind
        while (lanes < 6 && (1u << lanes) < chunks) ++lanes;
        if (T == 1 && chunks > 64) lanes = 8;                                     // one token: no others
        const unsigned groups = (chunks + (1u << lanes) - 1) >> lanes, tiles = (unsigned)((p.L + T - 1) / T);
        const size_t runs = ((size_t)tiles + (1u << (8 - lanes)) - 1) >> (8 - lanes);
        hipLaunchKernelGGL(kernel, dim3((unsigned)(runs * groups), (unsigned)p.batch), dim3(256), 0, stream, p, lanes, chunks, groups);
        return (int)hipGetLastError();
    };
    if (p.L == 1) return go(causal_conv_kernel<IO, VEC, 1, false>, 1);
    // Whatever comes next reads the outputs: they go through the caches as long as those can hold them (256 MB behind the L2s, which the
    // inputs pass too).  Conv and a sum over its outputs, us, through / past the caches: 34 MB 56.0 / 63.7, 84 MB 122.8 / 129.1,
    // 168 MB 277.7 / 270.4.
    // Four tokens of a thread: more of them in flight than with eight (us, 8 / 4: 100 x 8192 5.8 / 4.5, 2048 x 8192 14.7 / 13.9, 8 x 2048 x 5120
    // 62.4 / 60.8), but for large fp32 launches, which have enough of them (4 x 2048 x 8192: 95.7 / 99.5).
    constexpr int LONG = IO == SSMV_F32 ? 8 : 4;
    if constexpr (VEC > 1)
        if ((size_t)p.batch * p.L * p.C * Chunk<IO, VEC>::ES > (128u << 20)) return go(causal_conv_kernel<IO, VEC, LONG, true>, LONG);
    return go(causal_conv_kernel<IO, VEC, 4, false>, 4);
}

// a thread per element of conv_out
__global__ __launch_bounds__(256) void conv_history_kernel(const ConvHistoryParams p)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (size_t)p.batch * (W - 1) * p.Cx) return;
    const size_t row = i / p.Cx;
    const unsigned c = (unsigned)(i - row * p.Cx), b = (unsigned)(row / (W - 1)), k = (unsigned)(row - (size_t)b * (W - 1));
    const size_t at = ((size_t)b * p.R + ((p.conv_head[b] - (W - 2) + (int)k) & (p.R - 1))) * p.Cx + c;
    if (p.io == SSMV_BF16) static_cast<uint16_t *>(p.out)[i] = static_cast<const uint16_t *>(p.ring)[at];
    else static_cast<uint32_t *>(p.out)[i] = static_cast<const uint32_t *>(p.ring)[at];
}

}  // namespace

int launch_causal_conv(const CausalConvParams &p, hipStream_t stream)
{
    constexpr int EB = IoVec<SSMV_BF16>::EV, EF = IoVec<SSMV_F32>::EV;
    if (p.io == SSMV_BF16) return p.C >= EB ? launch<SSMV_BF16, EB>(p, stream) : launch<SSMV_BF16, 1>(p, stream);
    return p.C >= EF ? launch<SSMV_F32, EF>(p, stream) : launch<SSMV_F32, 1>(p, stream);
}

int launch_conv_history(const ConvHistoryParams &p, hipStream_t stream)
{
    const size_t n = (size_t)p.batch * (W - 1) * p.Cx;
    hipLaunchKernelGGL(conv_history_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream, p);
    return (int)hipGetLastError();
}

}  // namespace ssmv
