// A prompt through the recurrence with a decay per channel and state index, from state to state.
#include <type_traits>
#include <utility>

#include "decode_internal.h"

namespace ssmv {
namespace {

typedef float v4 __attribute__((ext_vector_type(4)));


// CH values of adjacent channels as stored; behind the last channel zeros
template <int IO, int CH>
struct Piece {
    static constexpr int NW = IO == SSMV_BF16 ? CH / 2 : CH;
    uint32_t w[NW];
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (IO == SSMV_BF16) return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else return __uint_as_float(w[i]);
    }
    // 8 or 16 bytes at the alignment of an element, but for the last channels of a row
    __device__ __forceinline__ void load(const char *from, int live)
    {
        if (live == CH) {
            __builtin_memcpy(w, from, sizeof(w));
        } else {
            uint32_t v[CH];
#pragma unroll
            for (int i = 0; i < CH; ++i) v[i] = i < live ? IoVec<IO>::load_raw1(from, i) : 0u;
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                if constexpr (IO == SSMV_BF16) w[i] = v[2 * i] | v[2 * i + 1] << 16;
                else w[i] = v[i];
            }
        }
    }
};

template <int IO, int CH>
__device__ __forceinline__ void store_piece(char *to, const float (&v)[CH], int live)
{
    if (live == CH) {
        uint32_t w[Piece<IO, CH>::NW];
#pragma unroll
        for (int i = 0; i < Piece<IO, CH>::NW; ++i) {
            if constexpr (IO == SSMV_BF16) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
            else w[i] = __float_as_uint(v[i]);
        }
        __builtin_memcpy(to, w, sizeof(w));
    } else {
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (i < live) store_io(to, i, v[i], IO);
    }
}

// the value that lane k of each 16 holds: an operand modifier of the multiplication that takes it
template <int K>
__device__ __forceinline__ float row_get(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x150 + K, 0xf, 0xf, true));
}

template <typename F, int... I>
__device__ __forceinline__ void unroll(F &&f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }

template <int S>
__device__ __forceinline__ void load_state(const float *from, float (&to)[S])
{
    if constexpr (S >= 4) {
#pragma unroll
        for (int i = 0; i < S; i += 4) {
            const v4 t = *reinterpret_cast<const v4 *>(from + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) to[i + j] = t[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < S; ++i) to[i] = from[i];
    }
}
template <int S>
__device__ __forceinline__ void store_state(float *to, const float (&from)[S])
{
    if constexpr (S >= 4) {
#pragma unroll
        for (int i = 0; i < S; i += 4) *reinterpret_cast<v4 *>(to + i) = v4{from[i], from[i + 1], from[i + 2], from[i + 3]};
    } else {
#pragma unroll
        for (int i = 0; i < S; ++i) to[i] = from[i];
    }
}

// (a, b) -> (rows 0, 1 of a | rows 0, 1 of b), (rows 2, 3 of a | rows 2, 3 of b), summed
__device__ __forceinline__ float fold32(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// the same of rows 0 and 1, and of rows 2 and 3
__device__ __forceinline__ float fold16(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The z-th longest of up to 64 sequences: workgroups start in the order of their indexes, and a long prompt that starts last leaves the
// chip to itself (8 ragged prompts x 5120: 248 -> 223 us).
__device__ __forceinline__ int by_length(const int32_t *seq_len, int batch, int z, unsigned lane)
{
    const int mine = (int)lane < batch ? seq_len[lane] : 0;
    int rank = 0;
    for (int i = 0; i < batch; ++i) {
        const int other = __builtin_amdgcn_readlane(mine, i);
        rank += other > mine || (other == mine && i < (int)lane);
    }
    return __builtin_ctzll(__ballot((int)lane < batch && rank == z));
}

constexpr int kScanWaves = 4, kHelpWaves = 4;

// h <- exp(dt' A) h + (dt' x) B,  y = C.h + D x: five operations and an exponential for every channel, token and state index, against 8 bytes
// (bf16, gated) for all N indices of a channel and token.  So the vector units bound it: an operation takes a wave 4 cycles, exp2 8, 24 in all;
// A and exp(dt' A) differ in every lane, which leaves the matrix cores nothing to contract but y, one useful column of sixteen.
//
// A workgroup takes CHW channels of a sequence, T tokens at a time.  Four of its waves scan: a lane per channel and S of the N state
// indices, which stay in registers from the first token to the last; with fewer than 64 channels the 64 / CHW parts of a wave take
// other indices of the same channels.  Four waves help: each of their threads owns CH adjacent channels of one token of a
// tile, prepares (dt', dt' x) of the tile ahead of the scan, and of the tile behind it sums the partial outputs, adds the skip, gates
// and stores, so that a tile's three stages run side by side and one barrier a tile is enough.  Everything changes hands in LDS.
// B of a token is a broadcast operand of the multiplication (16 / S tokens' worth sit in the lanes of every 16 of a register); as scalar
// registers B and C cost waits and unpacking on the scalar unit (522 us for 1 x 2048 x 8192 x 16, then in two barriers a tile, 225 with the broadcast).
// Measured, bf16, softplus and gate, us: 16 x 2048 x 8192 x 16 909, which is 34 cycles of a SIMD for 64 values of h (24 the recurrence, 3 its LDS
// accesses, 7 the helpers); 1 x 2048 x 8192 80 with the same inputs in every call, out of the caches (in workgroups of 64 channels 140, those in 8 segments
// 107), 85 with others, out of memory; 1 x 2048 x 1536 30 to 32 (in one segment 55); 8 x 2048 x 8192 x 64 1436.
// With 16 states a lane (N = 64 in workgroups of 64) the matrix cores add (dt' x) B, which for four channels and four state indices is a product of rank
// one: the 4 x 4 x 1 instruction takes a column of channels, the four lanes' B, and decay h to add to - exactly the lanes' own registers, and one
// instruction for four multiplications (8 x 2048 x 8192 x 64 1501 -> 1436, fp32 1498 -> 1456).  With eight states it made 1 % either way
// (8 x 2048 x 8192 x 32 782 -> 773, 1 x 2048 x 8192 x 64 252 -> 255) and with four nothing (16 x 2048 x 8192 x 16 910 -> 912): every token's then
// waits for the one before it.
// OUT false: only the state at the segment's end and the sum of its steps, of all segments but the last.
template <int IO, int N, int CHW, bool OUT>
__global__ __launch_bounds__(64 * (kScanWaves + kHelpWaves)) __attribute__((amdgpu_waves_per_eu(4)))
void selective_scan_kernel(const ScanParams p)
{
    constexpr int S = N * CHW / (64 * kScanWaves), R = 64 / CHW;                  // states of a lane; parts of a wave
    constexpr int CH = 4, T = 64 * kHelpWaves * CH / CHW, PER_ROW = CHW / CH, U = 4;
    constexpr int BC = 2 * T * N / (64 * kHelpWaves);                             // values of B and C that a thread fetches: of one token, adjacent
    constexpr int TB = S >= 16 ? 1 : 16 / S;                                      // tokens whose B share a register
    static_assert(S >= 1 && T % U == 0 && kScanTile % T == 0, "tile");
    __shared__ __attribute__((aligned(16))) float2 sIn[2][T][CHW];                // (dt', dt' x)
    __shared__ __attribute__((aligned(16))) float sB[2][T][N];
    __shared__ __attribute__((aligned(16))) float sC[2][OUT ? T : 1][N];
    __shared__ __attribute__((aligned(16))) float sY[2][kScanWaves][OUT ? T : 1][CHW];

    const unsigned lane = threadIdx.x & 63u;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned lin = xcd_contiguous(blockIdx.x, gridDim.x);                   // channels next to each other share cache lines
    const int c0 = (int)lin * CHW, seg = blockIdx.y;
    int b = blockIdx.z;
    if (p.seq_len && p.batch > 1 && p.batch <= 64) b = by_length(p.seq_len, p.batch, b, lane);
    const int all = p.seq_len ? min(max(p.seq_len[b], 0), p.L) : p.L;
    const int from = seg * p.seg_len, len = min(all, from + p.seg_len);           // the segment's tokens
    const bool last = len == all;
    if (OUT ? (seg > 0 && from >= all) : (seg > 0 && last)) return;
    const size_t slice = (size_t)p.C * N, tok0 = (size_t)b * p.L;
    float *seg_h = p.seg_h + (size_t)b * p.seg_count * slice;                     // the sequence's end states; the last place: where it starts

    if (wave < kScanWaves) {
        const int c = min(c0 + (int)(lane % CHW), p.C - 1);                       // lanes past the last channel double it and store nothing
        const bool have = c0 + (int)(lane % CHW) < p.C;
        const int n0 = (wave * R + (int)lane / CHW) * S;                          // the lane's state indices
        const size_t own = (size_t)c * N + n0;
        const float *seg_dt = p.seg_dt + (size_t)b * p.seg_count * p.C;
        float h[S], a[S];
        load_state<S>(p.A + own, a);
#pragma unroll
        for (int i = 0; i < S; ++i) { a[i] = decay_rate(a[i]); h[i] = 0.f; }
        if (seg == 0) {
            const int src = p.src_row ? p.src_row[b] : b;
            if (OUT && p.seg_count > 1) load_state<S>(seg_h + (p.seg_count - 1) * slice + own, h);    // h_out may be h_in, and its writer another workgroup
            else if (p.h_in && (unsigned)src < (unsigned)p.rows_in) load_state<S>(p.h_in + (size_t)src * slice + own, h);
            if (!OUT && have) store_state<S>(seg_h + (p.seg_count - 1) * slice + own, h);
        } else if (OUT) {
            load_state<S>(seg_h + own, h);
            for (int j = 1; j < seg; ++j) {
                float e[S];
                load_state<S>(seg_h + j * slice + own, e);
                const float sum = seg_dt[(size_t)j * p.C + c];
#pragma unroll
                for (int i = 0; i < S; ++i) h[i] = fmaf(h[i], __builtin_amdgcn_exp2f(a[i] * sum), e[i]);
            }
        }
        if (!OUT && last) return;                                                 // the whole workgroup: the helpers below, too
        float sum = 0.f;                                                          // of the lane's steps
        __syncthreads();
        for (int t0 = from, buf = 0; t0 < len; t0 += T, buf ^= 1) {
            const int n = min(len - t0, T);
            // U tokens at a time.  Of a whole tile the operands of the next U are requested ahead of the arithmetic on these where a lane has
            // few states: one wave a SIMD then waits for LDS otherwise (1 x 2048 x 8192 x 16: 92.9 -> 88.3 us).  With four states and
            // several waves a SIMD the registers that it takes cost more (16 x 2048 x 8192: 910 -> 936).
            struct Block {
                float2 in[U];
                float coef[S >= 16 ? U : (U + TB - 1) / TB], C[OUT ? U : 1][S];
            };
            auto load = [&](Block &k, int u0) {
#pragma unroll
                for (int u = 0; u < U; ++u) k.in[u] = sIn[buf][u0 + u][lane % CHW];
#pragma unroll
                for (int u = 0; u < U; u += TB)
                    k.coef[u / TB] = sB[buf][u0 + u + (S >= 16 ? 0 : ((int)lane % 16 / S) % U)][n0 + (int)lane % (S >= 16 ? 16 : S)];
                if constexpr (OUT)
#pragma unroll
                    for (int u = 0; u < U; ++u) load_state<S>(&sC[buf][u0 + u][n0], k.C[u]);
            };
            auto scan = [&](const Block &k, int u0) {
                float y[U];
                unroll([&](auto uu) {
                    constexpr int u = decltype(uu)::value;
                    y[u] = 0.f;
                    if constexpr (S >= 16) {
                        unroll([&](auto gg) {
                            constexpr int g = decltype(gg)::value;
                            v4 t;
#pragma unroll
                            for (int i = 0; i < 4; ++i) t[i] = h[4 * g + i] * __builtin_amdgcn_exp2f(a[4 * g + i] * k.in[u].x);
                            t = __builtin_amdgcn_mfma_f32_4x4x1f32(k.coef[u / TB], k.in[u].y, t, 2, g, 0);    // B of lanes 4g .. 4g + 3 of each 16
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                h[4 * g + i] = t[i];
                                if constexpr (OUT) y[u] = fmaf(k.C[u][4 * g + i], t[i], y[u]);
                            }
                        }, std::make_integer_sequence<int, S / 4>{});
                    } else {
                        unroll([&](auto ii) {
                            constexpr int i = decltype(ii)::value;
                            h[i] = fmaf(h[i], __builtin_amdgcn_exp2f(a[i] * k.in[u].x), row_get<u % TB * S + i>(k.coef[u / TB]) * k.in[u].y);
                            if constexpr (OUT) y[u] = fmaf(k.C[u][i], h[i], y[u]);
                        }, std::make_integer_sequence<int, S>{});
                    }
                    if constexpr (!OUT) sum += k.in[u].x;
                }, std::make_integer_sequence<int, U>{});
                if constexpr (OUT) {
#pragma unroll
                    for (int u = 0; u < U; u += R) {                              // part r of the wave ends up with token u + r
                        float v;
                        if constexpr (R == 1) v = y[u];
                        if constexpr (R == 2) v = fold32(y[u], y[u + 1]);
                        if constexpr (R == 4) v = fold16(fold32(y[u], y[u + 2]), fold32(y[u + 1], y[u + 3]));
                        sY[buf][wave][u0 + u + (int)lane / CHW][lane % CHW] = v;
                    }
                }
            };
            if (S <= 2 && n == T) {
                Block k[2];
                load(k[0], 0);
                unroll([&](auto bb) {
                    constexpr int blk = decltype(bb)::value;
                    if constexpr ((blk + 1) * U < T) load(k[(blk + 1) % 2], (blk + 1) * U);
                    __builtin_amdgcn_sched_barrier(0);
                    scan(k[blk % 2], blk * U);
                    __builtin_amdgcn_sched_barrier(0);
                }, std::make_integer_sequence<int, T / U>{});
            } else {
                for (int u0 = 0; u0 < n; u0 += U) {
                    Block k;
                    load(k, u0);
                    scan(k, u0);
                }
            }
            __syncthreads();
        }
        if (!have) return;
        if constexpr (OUT) {
            if (last && p.h_out) store_state<S>(p.h_out + (size_t)b * slice + own, h);
        } else {
            store_state<S>(seg_h + seg * slice + own, h);
            if (n0 == 0) p.seg_dt[((size_t)b * p.seg_count + seg) * p.C + c] = sum;
        }
        return;
    }

    if (!OUT && last) return;
    const int tid = (int)threadIdx.x - 64 * kScanWaves;
    const int row = tid / PER_ROW, col = tid % PER_ROW * CH, ch0 = c0 + col;
    const int live = min(max(p.C - ch0, 0), CH);                                  // channels that there are
    const int brow = tid * BC / (2 * N), bcol = tid * BC % (2 * N);               // the token of B and C, and where in that token's 2N values
    const bool is_c = bcol >= N;
    float bias[CH], D[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int at = min(ch0 + i, p.C - 1);
        bias[i] = p.dt_bias ? p.dt_bias[at] : 0.f;
        D[i] = OUT ? p.D[at] : 0.f;
    }
    const void *bc = is_c ? p.Cm : p.Bm;
    const size_t bc_stride = is_c ? p.c_stride : p.b_stride;
    constexpr int ES = IO == SSMV_BF16 ? 2 : 4, BCW = BC * ES / 4;
    struct Fetched {
        Piece<IO, CH> x, dt, z;
        uint32_t bc[BCW];
    } even, odd;                                                                  // of the next tiles but one: two are on their way
    Piece<IO, CH> px, pz, ex, ez;                                                 // of the tile being scanned; of the one behind it
    // where the thread's next pieces are: a tile further after every access
    const size_t tok = tok0 + from + row;
    const char *x_at = static_cast<const char *>(p.x) + (tok * p.x_stride + ch0) * ES, *dt_at = static_cast<const char *>(p.dt) + (tok * p.dt_stride + ch0) * ES;
    const char *z_at = static_cast<const char *>(p.z) + (tok * p.z_stride + ch0) * ES, *bc_at = static_cast<const char *>(bc) + ((tok0 + from + brow) * bc_stride + bcol % N) * ES;
    char *y_at = static_cast<char *>(p.y) + (tok * p.y_stride + ch0) * ES;
    auto fetch = [&](Fetched &f, int t0) {
        if (t0 >= len) return;
        const int n = t0 + row < len ? live : 0;                                  // what lies behind a sequence's tokens is not read
        f.x.load(x_at, n);
        f.dt.load(dt_at, n);
        if (OUT && p.z) f.z.load(z_at, n);
        const bool there = t0 + brow < len && (OUT || !is_c);
#pragma unroll
        for (int i = 0; i < BCW; ++i) f.bc[i] = there ? reinterpret_cast<const uint32_t *>(bc_at)[i] : 0u;
        x_at += T * ES * p.x_stride; dt_at += T * ES * p.dt_stride; z_at += T * ES * p.z_stride; bc_at += T * ES * bc_stride;
    };
    auto prepare = [&](const Fetched &f, int t0, int buf) {
        float2 in[CH];
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            float d = f.dt.get(i);
            if (p.softplus) d = softplus_exact(d + bias[i]);
            d = t0 + row < len ? d : 0.f;                                         // tokens that are none leave the state as it is
            in[i] = make_float2(d, d * f.x.get(i));
        }
#pragma unroll
        for (int i = 0; i < CH; i += 2) *reinterpret_cast<float4 *>(&sIn[buf][row][col + i]) = make_float4(in[i].x, in[i].y, in[i + 1].x, in[i + 1].y);
        if (OUT || !is_c) {
            float *to = is_c ? &sC[buf][OUT ? brow : 0][bcol % N] : &sB[buf][brow][bcol];
#pragma unroll
            for (int i = 0; i < BC; i += 2) {
                float2 v;
                if constexpr (IO == SSMV_BF16) v = make_float2(__uint_as_float(f.bc[i / 2] << 16), __uint_as_float(f.bc[i / 2] & 0xffff0000u));
                else v = make_float2(__uint_as_float(f.bc[i]), __uint_as_float(f.bc[i + 1]));
                *reinterpret_cast<float2 *>(to + i) = v;
            }
        }
    };
    auto finish = [&](int t0, int buf) {
        if (!OUT || t0 + row >= len) return;
        float y[CH];
        char *to = y_at;
        y_at += T * ES * p.y_stride;
#pragma unroll
        for (int i = 0; i < CH; ++i) y[i] = D[i] * ex.get(i);
#pragma unroll
        for (int w = 0; w < kScanWaves; ++w) {
            const v4 t = *reinterpret_cast<const v4 *>(&sY[buf][w][OUT ? row : 0][col]);
#pragma unroll
            for (int i = 0; i < CH; ++i) y[i] += t[i];
        }
        if (p.z)
#pragma unroll
            for (int i = 0; i < CH; ++i) y[i] *= silu_fast(ez.get(i));
        store_piece<IO, CH>(to, y, live);
    };
    fetch(even, from);
    fetch(odd, from + T);
    if (from < len) {
        prepare(even, from, 0);
        px = even.x; pz = even.z;
        fetch(even, from + 2 * T);
    }
    __syncthreads();
    int buf = 0, t0 = from;
    auto beside = [&](Fetched &f) {                                               // beside the scan of the tile at t0; f: of the next one
        if (t0 > from) finish(t0 - T, buf ^ 1);
        ex = px; ez = pz;
        if (t0 + T < len) {
            prepare(f, t0 + T, buf ^ 1);
            px = f.x; pz = f.z;
            fetch(f, t0 + 3 * T);
        }
        __syncthreads();
        t0 += T;
        buf ^= 1;
    };
    while (t0 < len) {
        beside(odd);
        if (t0 < len) beside(even);
    }
    if (t0 > from) finish(t0 - T, buf ^ 1);
}

template <int IO, int N, int CHW>
int launch(const ScanParams &p, hipStream_t stream)
{
    const unsigned blocks = (unsigned)((p.C + CHW - 1) / CHW);
    const dim3 block(64 * (kScanWaves + kHelpWaves)), ends(blocks, p.seg_count - 1, p.batch), all(blocks, p.seg_count, p.batch);
    if (p.seg_count > 1) {
        hipLaunchKernelGGL((selective_scan_kernel<IO, N, CHW, false>), ends, block, 0, stream, p);
        const int e = (int)hipGetLastError();
        if (e != 0) return e;
    }
    hipLaunchKernelGGL((selective_scan_kernel<IO, N, CHW, true>), all, block, 0, stream, p);
    return (int)hipGetLastError();
}

template <int IO, int N>
int launch_width(const ScanParams &p, hipStream_t stream)
{
    return p.channels_wg == 16 ? launch<IO, N, 16>(p, stream) : p.channels_wg == 32 ? launch<IO, N, 32>(p, stream) : launch<IO, N, 64>(p, stream);
}

template <int IO>
int launch_n(const ScanParams &p, hipStream_t stream)
{
    switch (p.N) {
        case 16: return launch_width<IO, 16>(p, stream);
        case 32: return launch_width<IO, 32>(p, stream);
        case 64: return launch_width<IO, 64>(p, stream);
    }
    return (int)hipErrorInvalidValue;
}

}  // namespace

int launch_selective_scan(const ScanParams &p, hipStream_t stream)
{
    return p.io == SSMV_BF16 ? launch_n<SSMV_BF16>(p, stream) : launch_n<SSMV_F32>(p, stream);
}

}  // namespace ssmv
