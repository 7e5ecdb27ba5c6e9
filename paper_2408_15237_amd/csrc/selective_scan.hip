// A prompt through the recurrence with a decay per channel and state index, from state to state.
#include "decode_internal.h"

namespace ssmv {
namespace {

typedef float v4 __attribute__((ext_vector_type(4)));

constexpr int kChannels = 64;            // channels of a workgroup: a lane each
constexpr int T = kScanTile;

// log(1 + e^v) for all v: max(v, 0) + log1p(t), t = e^-|v|, and log1p(t) = 2 atanh(s), s = t / (2 + t) <= 1/3, by its series up to s^13
// (what is left out is under 2^-25 of it).  No select, and no 1 + t that would lose the low bits of a small t.
__device__ __forceinline__ float softplus_series(float v)
{
    const float t = __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(v));
    const float s = t * __builtin_amdgcn_rcpf(2.f + t), q = s * s;
    float f = 2.f / 13.f;
    f = fmaf(f, q, 2.f / 11.f);
    f = fmaf(f, q, 2.f / 9.f);
    f = fmaf(f, q, 2.f / 7.f);
    f = fmaf(f, q, 2.f / 5.f);
    f = fmaf(f, q, 2.f / 3.f);
    f = fmaf(f, q, 2.f);
    return fmaf(s, f, fmaxf(v, 0.f));
}

// CH values of adjacent channels as stored; behind the last channel zeros
template <int IO, int CH>
struct Piece {
    static constexpr int NW = IO == SSMV_BF16 ? (CH + 1) / 2 : CH;
    uint32_t w[NW];
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (IO == SSMV_BF16) return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else return __uint_as_float(w[i]);
    }
    template <bool VEC>
    __device__ __forceinline__ void load(const void *base, size_t idx, int live)
    {
        if constexpr (VEC) {
            const uint32_t *s = reinterpret_cast<const uint32_t *>(static_cast<const char *>(base) + idx * (IO == SSMV_BF16 ? 2 : 4));
            if (live > 0) {
                if constexpr (NW >= 4) {
#pragma unroll
                    for (int i = 0; i < NW; i += 4) {
                        const uint4 t = *reinterpret_cast<const uint4 *>(s + i);
                        w[i] = t.x; w[i + 1] = t.y; w[i + 2] = t.z; w[i + 3] = t.w;
                    }
                } else if constexpr (NW == 2) {
                    const uint2 t = *reinterpret_cast<const uint2 *>(s);
                    w[0] = t.x; w[1] = t.y;
                } else {
                    w[0] = *s;
                }
            } else {
#pragma unroll
                for (int i = 0; i < NW; ++i) w[i] = 0;
            }
        } else {
            uint32_t v[CH];
#pragma unroll
            for (int i = 0; i < CH; ++i) v[i] = i < live ? IoVec<IO>::load_raw1(base, idx + i) : 0u;
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                if constexpr (IO == SSMV_BF16) w[i] = v[2 * i] | (2 * i + 1 < CH ? v[2 * i + 1] << 16 : 0u);
                else w[i] = v[i];
            }
        }
    }
};

template <int IO, int CH, bool VEC>
__device__ __forceinline__ void store_piece(void *base, size_t idx, const float (&v)[CH], int live)
{
    if constexpr (VEC) {
        if (live <= 0) return;
        constexpr int NW = Piece<IO, CH>::NW;
        uint32_t w[NW];
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            if constexpr (IO == SSMV_BF16) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
            else w[i] = __float_as_uint(v[i]);
        }
        uint32_t *d = reinterpret_cast<uint32_t *>(static_cast<char *>(base) + idx * (IO == SSMV_BF16 ? 2 : 4));
        if constexpr (NW >= 4) {
#pragma unroll
            for (int i = 0; i < NW; i += 4) *reinterpret_cast<uint4 *>(d + i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
        } else if constexpr (NW == 2) {
            *reinterpret_cast<uint2 *>(d) = make_uint2(w[0], w[1]);
        } else {
            d[0] = w[0];
        }
    } else {
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (i < live) store_io(base, idx + i, v[i], IO);
    }
}

// S state indices of a token's B or C, the same for all lanes: scalar loads
template <int IO, int S>
struct Coef {
    static constexpr int NW = IO == SSMV_BF16 ? S / 2 : S;
    uint32_t w[NW];
    __device__ __forceinline__ void load(const void *row)
    {
        const auto *s = (const __attribute__((address_space(4))) uint32_t *)(uintptr_t)row;
#pragma unroll
        for (int i = 0; i < NW; ++i) w[i] = s[i];
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (IO == SSMV_BF16) return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else return __uint_as_float(w[i]);
    }
};

// A workgroup takes 64 channels of a sequence, T tokens at a time: a lane per channel, a wave per S state indices, so that B and C of
// a token are wave-uniform (scalar registers) and a lane's state stays in registers from the first token to the last.  Around the
// recurrence every thread owns CH adjacent channels of one token of the tile: it prepares (dt', dt' x) for the waves, and sums their
// partial outputs, adds the skip, gates and stores.  Both change hands in LDS.
template <int IO, int N, int S, bool VEC>
__global__ __launch_bounds__(64 * (N / S)) void selective_scan_kernel(const ScanParams p)
{
    constexpr int NW = N / S, THREADS = 64 * NW, CH = T * kChannels / THREADS, PER_ROW = kChannels / CH, U = 8;
    constexpr float LOG2E = 1.4426950408889634f;
    __shared__ __attribute__((aligned(16))) float2 sIn[T][kChannels];             // (dt', dt' x)
    __shared__ __attribute__((aligned(16))) float sY[NW][T][kChannels];

    const unsigned tid = threadIdx.x, lane = tid & 63u;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const unsigned blocks = gridDim.x;
    const unsigned lin = xcd_contiguous(blockIdx.y * blocks + blockIdx.x, blocks * gridDim.y);
    const int b = __builtin_amdgcn_readfirstlane(lin / blocks), c0 = (int)(lin - (unsigned)b * blocks) * kChannels;
    const int len = p.seq_len ? min(max(p.seq_len[b], 0), p.L) : p.L;

    // the lane's part of the state
    const int c = min(c0 + (int)lane, p.C - 1);                                   // lanes past the last channel double it and store nothing
    const bool have = c0 + (int)lane < p.C;
    const int src = p.src_row ? p.src_row[b] : b;
    const size_t own = (size_t)c * N + wave * S;
    float h[S], a[S];
#pragma unroll
    for (int i = 0; i < S; i += 4) {
        const v4 t = *reinterpret_cast<const v4 *>(p.A + own + i) * LOG2E;
        v4 s = v4{0.f, 0.f, 0.f, 0.f};
        if (p.h_in && (unsigned)src < (unsigned)p.rows_in) s = *reinterpret_cast<const v4 *>(p.h_in + (size_t)src * p.C * N + own + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) { a[i + j] = t[j]; h[i + j] = s[j]; }
    }

    // the thread's part of a tile
    const int row = (int)tid / PER_ROW, col = (int)(tid % PER_ROW) * CH, ch0 = c0 + col;
    const int live = min(max(p.C - ch0, 0), CH);                                  // channels that there are
    float bias[CH], D[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int at = min(ch0 + i, p.C - 1);
        bias[i] = p.dt_bias ? p.dt_bias[at] : 0.f;
        D[i] = p.D[at];
    }
    const size_t tok0 = (size_t)b * p.L;
    Piece<IO, CH> x, dt, z, nx, ndt, nz;
    auto fetch = [&](int t0, Piece<IO, CH> &px, Piece<IO, CH> &pdt, Piece<IO, CH> &pz) {
        const int n = t0 + row < len ? live : 0;                                  // what lies behind a sequence's tokens is not read
        const size_t tok = tok0 + t0 + row;
        px.template load<VEC>(p.x, tok * p.x_stride + ch0, n);
        pdt.template load<VEC>(p.dt, tok * p.dt_stride + ch0, n);
        if (p.z) pz.template load<VEC>(p.z, tok * p.z_stride + ch0, n);
    };
    if (len > 0) fetch(0, nx, ndt, nz);

    for (int t0 = 0; t0 < len; t0 += T) {
        const int n = min(len - t0, T);
        x = nx; dt = ndt; z = nz;
        {
            float2 in[CH];
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                float d = dt.get(i);
                if (p.softplus) d = softplus_series(d + bias[i]);
                d = row < n ? d : 0.f;                                            // tokens that are none leave the state as it is
                in[i] = make_float2(d, d * x.get(i));
            }
#pragma unroll
            for (int i = 0; i < CH; i += 2) *reinterpret_cast<float4 *>(&sIn[row][col + i]) = make_float4(in[i].x, in[i].y, in[i + 1].x, in[i + 1].y);
        }
        __syncthreads();
        if (t0 + T < len) fetch(t0 + T, nx, ndt, nz);
        const int e = IO == SSMV_BF16 ? 2 : 4;
        for (int u0 = 0; u0 < n; u0 += U) {
            Coef<IO, S> B[U], C[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const size_t tok = tok0 + min(t0 + u0 + u, len - 1);
                B[u].load(static_cast<const char *>(p.Bm) + (tok * p.b_stride + wave * S) * e);
                C[u].load(static_cast<const char *>(p.Cm) + (tok * p.c_stride + wave * S) * e);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float2 in = sIn[u0 + u][lane];
                float y = 0.f;
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    h[i] = fmaf(h[i], __builtin_amdgcn_exp2f(a[i] * in.x), in.y * B[u].get(i));
                    y = fmaf(h[i], C[u].get(i), y);
                }
                sY[wave][u0 + u][lane] = y;
            }
        }
        __syncthreads();
        if (row < n) {
            float y[CH];
#pragma unroll
            for (int i = 0; i < CH; ++i) y[i] = D[i] * x.get(i);
#pragma unroll
            for (int w = 0; w < NW; ++w)
#pragma unroll
                for (int i = 0; i < CH; ++i) y[i] += sY[w][row][col + i];
            if (p.z)
#pragma unroll
                for (int i = 0; i < CH; ++i) y[i] *= silu_fast(z.get(i));
            store_piece<IO, CH, VEC>(p.y, (tok0 + t0 + row) * p.y_stride + ch0, y, live);
        }
    }
    if (p.h_out && have)
#pragma unroll
        for (int i = 0; i < S; i += 4) *reinterpret_cast<v4 *>(p.h_out + (size_t)b * p.C * N + own + i) = v4{h[i], h[i + 1], h[i + 2], h[i + 3]};
}

template <int IO, int N, int S>
int launch(const ScanParams &p, hipStream_t stream)
{
    const dim3 grid((unsigned)((p.C + kChannels - 1) / kChannels), (unsigned)p.batch), block(64 * (N / S));
    if (p.vec) hipLaunchKernelGGL((selective_scan_kernel<IO, N, S, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((selective_scan_kernel<IO, N, S, false>), grid, block, 0, stream, p);
    return (int)hipGetLastError();
}

template <int IO>
int launch_n(const ScanParams &p, hipStream_t stream)
{
    switch (p.N) {
        case 16: return launch<IO, 16, 4>(p, stream);
        case 32: return launch<IO, 32, 8>(p, stream);
        case 64: return launch<IO, 64, 8>(p, stream);
    }
    return (int)hipErrorInvalidValue;
}

}  // namespace

int launch_selective_scan(const ScanParams &p, hipStream_t stream)
{
    return p.io == SSMV_BF16 ? launch_n<SSMV_BF16>(p, stream) : launch_n<SSMV_F32>(p, stream);
}

}  // namespace ssmv
