// What the forward and the backward pass of the gated recurrence share: how lanes lie over channels and tokens, the loads of a tile, and how the runs of a wave combine.
#pragma once

#include "layers_internal.h"

namespace ssmv {

constexpr int kRun = 4;      // tokens that a lane takes one after the other

// A lane owns 4 bytes of a token's row (two bf16 channels, one fp32) for kRun tokens: lane l of a wave the channels l % CL and the run l / CL.
// The last channels of a row are a pair moved back, whose first `skip` channels are another lane's; lanes behind the row have skip >= CH, load what others load and store nothing.
template <int IO, int CL>
struct GatedLane {
    static constexpr int CH = IO == SSMV_BF16 ? 2 : 1, ES = IO == SSMV_BF16 ? 2 : 4;
    static constexpr int CW = CL * CH;                         // channels of a workgroup
    static constexpr int RUNS = 64 / CL, WT = RUNS * kRun;     // runs and tokens of a wave

    int c0, skip, C;
    __device__ __forceinline__ GatedLane(int own, int channels) : c0(max(min(own, channels - CH), 0)), skip(own - c0), C(channels) {}
    __device__ __forceinline__ bool mine(int c) const { return c >= skip && c0 + c < C; }
    __device__ __forceinline__ int channel(int c) const { return min(c0 + c, C - 1); }

    static __device__ __forceinline__ void decode(uint32_t w, float (&v)[CH])
    {
        if constexpr (IO == SSMV_BF16) {
            v[0] = __uint_as_float(w << 16);
            v[1] = __uint_as_float(w & 0xffff0000u);
        } else {
            v[0] = __uint_as_float(w);
        }
    }
    static __device__ __forceinline__ uint32_t encode(const float (&v)[CH])
    {
        if constexpr (IO == SSMV_BF16) return pack_bf16x2(v[0], v[CH - 1]);
        else return __float_as_uint(v[0]);
    }
    // of a row of at least CH channels
    static __device__ __forceinline__ uint32_t load(const char *at)
    {
        uint32_t r;
        __builtin_memcpy(&r, at, 4);
        return r;
    }
    static __device__ __forceinline__ void store(char *at, uint32_t r) { __builtin_memcpy(at, &r, 4); }
    static __device__ __forceinline__ void store_past(char *at, uint32_t r)          // past the caches
    {
        typedef uint32_t loose __attribute__((aligned(2)));
        __builtin_nontemporal_store(r, reinterpret_cast<loose *>(at));
    }
    // any row
    __device__ __forceinline__ uint32_t load_any(const char *row) const
    {
        if (C >= CH) return load(row + (size_t)c0 * ES);
        return *reinterpret_cast<const uint16_t *>(row);
    }
    __device__ __forceinline__ void store_any(char *row, const float (&v)[CH]) const
    {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (mine(c)) store_io(row, c0 + c, v[c], IO);
    }
    __device__ __forceinline__ void floats(const float *from, float (&v)[CH]) const
    {
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c] = from[channel(c)];
    }
    __device__ __forceinline__ void put_floats(float *to, const float (&v)[CH]) const
    {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (mine(c)) to[c0 + c] = v[c];
    }
};

// 4 bytes per lane from global memory straight into LDS: lane l's word lands at `dst` + 4 l (the same in all lanes; it travels in M0).  Issued from assembly, so that the
// compiler does not wait for it at its next LDS read; the kernel waits by itself (vmcnt).  The base is copied by a scalar instruction, which waits for a vector instruction that
// wrote it (a vector memory access would need five wait states) and is the wait state that M0 asks for.
typedef __attribute__((address_space(3))) char lds_byte;
__device__ __forceinline__ void load_to_lds(const char *base, unsigned offset, const uint32_t *dst)
{
    const unsigned lds_addr = (unsigned)(size_t)(lds_byte *)dst;
    const char *copy;
    asm volatile("s_mov_b32 m0, %3\n\ts_mov_b64 %0, %2\n\tglobal_load_lds_dword %1, %0" : "=&s"(copy) : "v"(offset), "s"(base), "s"(lds_addr) : "memory", "m0");
}
// until at most COUNT of the wave's memory accesses are under way
template <int COUNT>
__device__ __forceinline__ void wait_but() { asm volatile("s_waitcnt vmcnt(%0)" ::"i"(COUNT) : "memory"); }

// The value is worked out here: the compiler may not keep its operands instead and finish it where it is used, which costs a register for each of them.
__device__ __forceinline__ void settle(float &v) { asm volatile("" : "+v"(v)); }

// One tensor of tokens, as a wave walks through it tile by tile: `at` is the wave's first token of a tile.
template <int IO, int CL>
struct Walk {
    using Ln = GatedLane<IO, CL>;
    const char *at;
    uint32_t step;           // bytes between tokens
    unsigned off;            // of the lane's run and channels from `at`
    __device__ __forceinline__ Walk(const void *base, size_t stride, size_t token, unsigned run, const Ln &ln)
        : at(static_cast<const char *>(base) + token * stride * Ln::ES), step((uint32_t)stride * Ln::ES), off((run * kRun * (unsigned)stride + (unsigned)ln.c0) * Ln::ES) {}
    __device__ __forceinline__ void move(int tokens) { at += (ptrdiff_t)tokens * (ptrdiff_t)step; }
    // the run's tokens, all of them there
    __device__ __forceinline__ void load(uint32_t (&r)[kRun]) const
    {
        const char *row = at;
        unsigned o = off;
        asm volatile("" : "+v"(o));     // stays a 32-bit offset from a scalar base
#pragma unroll
        for (int k = 0; k < kRun; ++k, row += step) r[k] = Ln::load(row + o);
    }
    // into LDS: the k-th token's words `each` apart
    __device__ __forceinline__ void prefetch(const uint32_t *dst, int each) const
    {
        const char *row = at;
#pragma unroll
        for (int k = 0; k < kRun; ++k, row += step) load_to_lds(row, off, dst + k * each);
    }
    // t: the token at `at`; tokens from `len` on are the last one again
    __device__ __forceinline__ void load_tail(uint32_t (&r)[kRun], int t, unsigned run, int len, const Ln &ln) const
    {
        const char *row[kRun];
#pragma unroll
        for (int k = 0; k < kRun; ++k) row[k] = at + (ptrdiff_t)(min(t + (int)run * kRun + k, len - 1) - t) * (ptrdiff_t)step;
        if (Ln::CH == 1 || ln.C >= Ln::CH) {
#pragma unroll
            for (int k = 0; k < kRun; ++k) r[k] = Ln::load(row[k] + (size_t)ln.c0 * Ln::ES);
        } else {
#pragma unroll
            for (int k = 0; k < kRun; ++k) r[k] = *reinterpret_cast<const uint16_t *>(row[k]);
        }
    }
    template <bool TAIL>
    __device__ __forceinline__ void store(const float (&v)[kRun][Ln::CH], int t, unsigned run, int len, const Ln &ln, bool past) const
    {
        char *row = const_cast<char *>(at);
        if constexpr (!TAIL) {
            uint32_t r[kRun];
#pragma unroll
            for (int k = 0; k < kRun; ++k) r[k] = Ln::encode(v[k]);
            if (ln.skip == 0) {
                if (past) {
#pragma unroll
                    for (int k = 0; k < kRun; ++k, row += step) Ln::store_past(row + off, r[k]);
                } else {
#pragma unroll
                    for (int k = 0; k < kRun; ++k, row += step) Ln::store(row + off, r[k]);
                }
            } else if (ln.skip < Ln::CH) {                          // the second of two channels
#pragma unroll
                for (int k = 0; k < kRun; ++k, row += step) *reinterpret_cast<uint16_t *>(row + off + 2) = (uint16_t)(r[k] >> 16);
            }
        } else {
            row += (size_t)(run * kRun) * step;
            const bool both = ln.skip == 0 && ln.C >= Ln::CH;
#pragma unroll
            for (int k = 0; k < kRun; ++k, row += step) {
                if (t + (int)run * kRun + k >= len) continue;
                if (both) Ln::store(row + (size_t)ln.c0 * Ln::ES, Ln::encode(v[k]));
                else ln.store_any(row, v[k]);
            }
        }
    }
};

// The value that the even, and the odd, row of 16 lanes of each pair holds, in both rows; the same of the halves of a wave.
__device__ __forceinline__ void rows_of_pair(float v, float &even, float &odd)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    even = __uint_as_float(r[0]);
    odd = __uint_as_float(r[1]);
}
__device__ __forceinline__ void halves(float v, float &low, float &high)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    low = __uint_as_float(r[0]);
    high = __uint_as_float(r[1]);
}

// (P, H) of the 64 / CL runs of a wave, first to last: that of the runs before the lane's, and of all, in every lane.
template <int CL>
__device__ __forceinline__ void combine_forward(float P, float H, unsigned run, float &Pe, float &He, float &Pt, float &Ht)
{
    float p0, p1, h0, h1;
    if constexpr (CL == 32) {
        halves(P, p0, p1);
        halves(H, h0, h1);
        Pt = p0 * p1;
        Ht = fmaf(p1, h0, h1);
        Pe = run ? p0 : 1.f;
        He = run ? h0 : 0.f;
    } else {
        static_assert(CL == 16, "lanes");
        rows_of_pair(P, p0, p1);
        rows_of_pair(H, h0, h1);
        float pa, pb, ha, hb;                                  // of the first and of the second pair
        halves(p0 * p1, pa, pb);
        halves(fmaf(p1, h0, h1), ha, hb);
        Pt = pa * pb;
        Ht = fmaf(pb, ha, hb);
        const bool odd = run & 1, second = run & 2;
        const float pr = odd ? p0 : 1.f, hr = odd ? h0 : 0.f;   // the run before in the lane's pair
        Pe = second ? pa * pr : pr;
        He = second ? fmaf(pr, ha, hr) : hr;
    }
}
// (P, R) from the last run to the first: that of the runs behind the lane's, and R of all (the product of all is the forward one's).
template <int CL>
__device__ __forceinline__ void combine_backward(float P, float R, unsigned run, float &Pe, float &Re, float &Rt)
{
    float p0, p1, r0, r1;
    if constexpr (CL == 32) {
        halves(P, p0, p1);
        halves(R, r0, r1);
        Rt = fmaf(p0, r1, r0);
        Pe = run ? 1.f : p1;
        Re = run ? 0.f : r1;
    } else {
        static_assert(CL == 16, "lanes");
        rows_of_pair(P, p0, p1);
        rows_of_pair(R, r0, r1);
        float pa, pb, ra, rb;
        halves(p0 * p1, pa, pb);
        halves(fmaf(p0, r1, r0), ra, rb);
        Rt = fmaf(pa, rb, ra);
        const bool odd = run & 1, second = run & 2;
        const float pr = odd ? 1.f : p1, rr = odd ? 0.f : r1;
        Pe = second ? pr : pb * pr;
        Re = second ? rr : fmaf(pr, rb, rr);
    }
}

}  // namespace ssmv
