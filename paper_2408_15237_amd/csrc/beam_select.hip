// Beam search's choice over all beams and the vocabulary.
#include "decode_internal.h"

namespace ssmv {
namespace {

typedef unsigned long long Key;
constexpr float kTop = 3.402823466e+38f;                                        // the largest finite value

// A candidate of a row as a whole number: larger is better - the logit in an order-preserving form above, the token's
// complement below, so that keys are unique and equal logits go by the lower token.  0 stands for none.
__device__ __forceinline__ Key key_of(float v, unsigned token)
{
    unsigned u = __float_as_uint(v + 0.f);                                        // -0 + 0 = 0
    u = u & 0x80000000u ? ~u : u | 0x80000000u;
    return (Key)u << 32 | (0xffffffffu - token);
}
__device__ __forceinline__ float key_logit(Key k)
{
    const unsigned u = (unsigned)(k >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ unsigned key_token(Key k) { return 0xffffffffu - (unsigned)k; }

// v combined over the wave, with the lanes 1, 2, 4, .. apart (lanes of each other half) and without a trip through LDS
template <int CTRL>
__device__ __forceinline__ float dpp(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true)); }
template <typename F>
__device__ __forceinline__ float combine(float v, F &&f)                          // f(one, other, how many lanes apart)
{
    v = f(v, dpp<0xB1>(v), 1);                                                    // the other lane of a pair, the other pair of a quad
    v = f(v, dpp<0x4E>(v), 2);
    v = f(v, dpp<0x141>(v), 4);                                                   // mirrored in 8, in 16
    v = f(v, dpp<0x140>(v), 8);
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(r[0]), __uint_as_float(r[1]), 16);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]), 32);
}
// the largest of the lanes that are alike modulo `apart`, 1 or 2
__device__ __forceinline__ float alike(float v, int apart)
{
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    v = fmaxf(v, dpp<0x128>(v));                                                  // 16 lanes rotated by 8, 4, 2, 1
    v = fmaxf(v, dpp<0x124>(v));
    v = fmaxf(v, dpp<0x122>(v));
    return apart == 1 ? fmaxf(v, dpp<0x121>(v)) : v;
}
// the sum over the wave, in 64 bits
__device__ __forceinline__ double wave_sum64(double v)
{
    auto both = [&](auto &&move) {
        const unsigned long long b = __builtin_bit_cast(unsigned long long, v);
        const unsigned lo = __float_as_uint(move(__uint_as_float((unsigned)b))), hi = __float_as_uint(move(__uint_as_float((unsigned)(b >> 32))));
        v += __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
    };
    both([](float x) { return dpp<0xB1>(x); });
    both([](float x) { return dpp<0x4E>(x); });
    both([](float x) { return dpp<0x141>(x); });
    both([](float x) { return dpp<0x140>(x); });
    auto swapped = [&](auto &&swap) {
        const unsigned long long b = __builtin_bit_cast(unsigned long long, v);
        const auto lo = swap((unsigned)b), hi = swap((unsigned)(b >> 32));
        v = __builtin_bit_cast(double, (unsigned long long)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (unsigned long long)hi[1] << 32 | lo[1]);
    };
    swapped([](unsigned x) { return __builtin_amdgcn_permlane16_swap(x, x, false, false); });
    swapped([](unsigned x) { return __builtin_amdgcn_permlane32_swap(x, x, false, false); });
    return v;
}
__device__ __forceinline__ double lane_get(double v, int lane)
{
    const unsigned long long b = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = __builtin_amdgcn_readlane((unsigned)b, lane), hi = __builtin_amdgcn_readlane((unsigned)(b >> 32), lane);
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
__device__ __forceinline__ float larger(float a, float b, int) { return fmaxf(a, b); }
__device__ __forceinline__ float sum_of(float a, float b, int) { return a + b; }

constexpr int THREADS = 256, WAVES = THREADS / 64, PAIRS = THREADS / 2;
// Up to so many candidates a bound of group maxima is as good as any; of more, the least of as many groups lets too many pass (us of a piece,
// groups / the pairs' `keep`-th: 224 rows of 1318, 16 6.6 / 5.6, 32 14.9 / 7.1, 64 38 / 10)
constexpr int kFewKeep = 2 * WAVES;
// Up to so many candidates of a sequence the largest of the rows' last scores bounds the choice (us of the merge, this bound / the other one:
// 3 rows of 6 4.9 / 5.6, 16 of 16 7.4 / 7.8, 16 of 32 10.6 / 8.2, 16 of 64 26 / 10.6)
constexpr int kFewCandidates = 256;
constexpr int kList = 1024;                                                       // candidates that the short way of a piece may collect

// Logits are read once, and that is the least a selection can do; beside it stand a row's sum (an exponential for every logit) and
// its best candidates.
//
// The best `keep` candidates of a piece of a row, best first, and its part of the row's sum; E logits of a thread at a time.
// A bound that at least `keep` logits reach: the least of the largest logits of `keep` groups of lanes, or of many the `keep`-th largest of the
// pairs of lanes (kFewKeep).  What reaches it is collected and ranked - some tens of candidates.  Where ties make them too many, the
// bound is taken of the threads' best keys, which are unique: only the `keep` threads at or above it can hold any candidate, keep * E at most.
// A row may begin anywhere: its vectors are read where its own elements lie (16 bytes at the alignment of an element), so that which
// thread takes a token, and with it the order of the sum, does not depend on the address, and equal rows stay equal to the last bit.
// Measured: 16 x 8 rows of 128011 bf16 (33 MB) 13.7 us, of which loads and maxima alone take 6.4, the exponentials 1.7, collecting and
// ranking 4 (vector instructions 6.0 in all, waits half of the waves' time); then 4.9 for the merge.  128 x 8 rows 72 us,
// 3.6 TB/s, vector instructions 43.  (All candidates ranked against all threads' best and lists merged by binary searches: 68 us.  One workgroup for
// all of a sequence, in one launch: 12.7 us for one row of 32000, where two launches take 8.3.)
template <int IO, int E>
__global__ __launch_bounds__(THREADS) void beam_piece_kernel(const BeamParams p)
{
    constexpr int EV = IoVec<IO>::EV, CHUNK = THREADS * E, ES = IO == SSMV_BF16 ? 2 : 4;
    constexpr int kMost = (E > 8 ? SSMV_BEAMS_MAX : kSmallKeep) * E;              // of the long way; the list has room for both
    constexpr float LOG2E = 1.4426950408889634f;
    __shared__ Key sList[kList + kMost];
    __shared__ Key sBest[SSMV_BEAMS_MAX], sThread[THREADS];
    __shared__ __attribute__((aligned(16))) float sMax[PAIRS];
    __shared__ float sSum[WAVES], sLeast[2], sTop[2];
    __shared__ Key sKey;
    __shared__ int sCount;
    const unsigned tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    const int piece = blockIdx.x, keep = p.keep;
    const size_t row = blockIdx.y;
    const int done = p.done ? p.done[row] : 0;
    const char *base = static_cast<const char *>(p.logits) + row * p.row_stride * ES;
    Key *out = p.keys + (row * p.pieces + piece) * keep;
    const int own = keep <= WAVES ? 1 : 2;                                            // groups of a wave: lanes alike modulo `own`

    const int begin = piece * p.piece_len, end = min(p.V, begin + p.piece_len);
    float m = -kTop, sum = 0.f, bound = -INFINITY;                                // of the chunks so far
    // A thread's vectors of a chunk, all requested before the first is used, and a chunk ahead of its arithmetic.  The waves have equal
    // shares of the chunk's vectors, a row's end too, so that no group is left with few.  A vector that reaches past the
    // end is moved back to it: the tokens ahead of its own place, which are another vector's, hold -inf then.
    uint4 raw[E / EV];
    auto share = [&](int first) { return (min(CHUNK / EV, (end - first + EV - 1) / EV) + WAVES - 1) / WAVES; };
    auto vector = [&](int first, int q, int i) {                                  // where the i-th begins; the end where there is none
        const int l = i * 64 + (int)lane;
        return l < q ? first + ((int)wave * q + l) * EV : end;
    };
    auto fetch = [&](int first) {
        const int q = share(first);
#pragma unroll
        for (int i = 0; i < E / EV; ++i) {
            const int at = min(vector(first, q, i), end - EV);
            __builtin_memcpy(&raw[i], base + (ptrdiff_t)at * ES, sizeof(uint4));
        }
    };
    if (end >= EV) fetch(begin);
    if (done != 0) return;                                                        // a finished row: known by when the first logits are on their way
    if (tid == 0) sCount = 0;
    // the places of the list's first `count` keys: a quad of lanes to a key
    auto rank = [&](int count, Key *to) {
        for (int i = tid / 4; i < count; i += THREADS / 4) {
            const Key k = sList[i];
            int r = 0;
#pragma unroll 4
            for (int j = tid % 4; j < count; j += 4) r += sList[j] > k;
            r += __shfl_xor(r, 1);
            r += __shfl_xor(r, 2);
            if (r < keep && tid % 4 == 0) to[r] = k;
        }
    };
    for (int chunk = 0; chunk < p.chunks; ++chunk) {
        const int first = begin + chunk * CHUNK;
        const int q = share(first);
        auto place = [&](int i) { return vector(first, q, i / EV); };
        auto pos = [&](int i) { return min(place(i), end - EV) + i % EV; };
        auto there = [&](int i) { return pos(i) >= place(i); };
        float v[E];
        if (end >= EV) {
#pragma unroll
            for (int i = 0; i < E / EV; ++i) {
                float d[EV];
                IoVec<IO>::decode(raw[i], d);
#pragma unroll
                for (int j = 0; j < EV; ++j) v[i * EV + j] = d[j];
            }
            if (first + CHUNK > end) {
#pragma unroll
                for (int i = 0; i < E; i += EV)
                    if (place(i) > end - EV) {
#pragma unroll
                        for (int j = i; j < i + EV; ++j) v[j] = there(j) ? v[j] : -INFINITY;
                    }
            }
            if (chunk + 1 < p.chunks) fetch(first + CHUNK);
        } else {                                                                  // a vocabulary of less than one vector
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = i < EV && there(i) && pos(i) >= 0 ? load_io(base, (size_t)pos(i), IO) : -INFINITY;
        }
        float most = -INFINITY;                                                   // (the maximum of a number and NaN is the number)
#pragma unroll
        for (int i = 0; i < E; ++i) most = fmaxf(most, v[i]);
        const float before = m;
        float least = INFINITY;
        if (keep <= kFewKeep) {
            const float group = alike(most, own);
            if (lane < (unsigned)own) sMax[wave * own + lane] = group;
            __syncthreads();
            for (int g = 0; g < WAVES * own; g += 4) {
                const float4 t = *reinterpret_cast<const float4 *>(sMax + g);
                m = fmaxf(fmaxf(fmaxf(m, t.x), fmaxf(t.y, t.z)), t.w);
                least = fminf(fminf(least, t.x), fminf(fminf(t.y, t.z), t.w));
            }
        } else {
            const float pair = fmaxf(most, dpp<0xB1>(most));
            if (tid % 2 == 0) sMax[tid / 2] = pair;
            __syncthreads();
            if (tid < PAIRS) {
                const float mine = sMax[tid];
                int above = 0;
#pragma unroll 4
                for (int g = 0; g < PAIRS; g += 4) {
                    const float4 t = *reinterpret_cast<const float4 *>(sMax + g);
                    above += (t.x > mine) + (t.y > mine) + (t.z > mine) + (t.w > mine);
                }
                const float low = combine(above < keep ? mine : INFINITY, [](float a, float b, int) { return fminf(a, b); }), top = combine(mine, larger);
                if (lane == 0) { sLeast[wave] = low; sTop[wave] = top; }
            }
            __syncthreads();
            least = fminf(sLeast[0], sLeast[1]);
            m = fmaxf(m, fmaxf(sTop[0], sTop[1]));
        }
        if (m == INFINITY) {                                                      // +inf is the largest finite logit
            m = kTop;
            least = fminf(least, kTop);
            most = fminf(most, kTop);
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = v[i] == INFINITY ? kTop : v[i];
        }
        bound = fmaxf(bound, least);
        const int held = sCount;                                                  // candidates of the chunks before
        const bool open = bound == -INFINITY;                                     // a group without a token that is allowed
        __syncthreads();
        unsigned hits = 0;
        int at = 0, near[2] = {0, 0};
        float logit[2] = {0.f, 0.f};
        auto token = [&](unsigned bits) {                                         // of the lowest set bit
            const int i = E - 1 - __builtin_ctz(bits);
            return pos(i);
        };
        if (!open && most >= bound) {
#pragma unroll
            for (int i = 0; i < E; ++i) hits = 2 * hits + (v[i] >= bound);
            at = atomicAdd(&sCount, __builtin_popcount(hits));
            near[0] = token(hits);
            near[1] = hits & (hits - 1) ? token(hits & (hits - 1)) : near[0];
#pragma unroll
            for (int k = 0; k < 2; ++k) logit[k] = load_io(base, (size_t)near[k], IO);    // once more, out of the cache; back by when the sum is done
        }
        // exp(v - m) as one fused operation and exp2: the reference is what m log2 e rounds to, and the sum is corrected for that.  Up to 2^20 the
        // rounding is 2^-4 at most; of a larger m the terms would move by its powers of two (a row masked by -1e10: to 0 or infinity), so the
        // difference comes first
        const bool far = fabsf(m) > 1048576.f;
        const float ref = far ? 0.f : m * LOG2E;
        auto total = [&]() {
            float t = 0.f;
            if (far) {
#pragma unroll
                for (int i = 0; i < E; ++i) t += __builtin_amdgcn_exp2f((v[i] - m) * LOG2E);
                return t;
            }
#pragma unroll
            for (int i = 0; i < E; ++i) t += __builtin_amdgcn_exp2f(fmaf(v[i], LOG2E, -ref));
            return t * __builtin_amdgcn_exp2f(-fmaf(m, LOG2E, -ref));
        };
        float part = total();
        if (part != part) {                                                       // NaN is a token that is not allowed
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = v[i] != v[i] ? -INFINITY : v[i];
            part = total();
        }
        sum = fmaf(sum, __builtin_amdgcn_exp2f((before - m) * LOG2E), part);
        for (int k = 0; hits && at < kList; ++k) {                                // one, hardly ever more than two
            if (k >= 2) {
                near[1] = token(hits);
                logit[1] = load_io(base, (size_t)near[1], IO);
            }
            const float l = k == 0 ? logit[0] : logit[1];
            sList[at++] = key_of(l == INFINITY ? kTop : l, (unsigned)(k == 0 ? near[0] : near[1]));
            hits &= hits - 1;
        }
        const bool final = chunk + 1 == p.chunks;
        if (final) {
            const float all = combine(sum, sum_of);
            if (lane == 0) sSum[wave] = all;
        }
        __syncthreads();
        int count = sCount;
        if (open || count > kList) {                                              // the same for all threads
            Key best = 0;
#pragma unroll
            for (int i = 0; i < E; ++i)
                if (there(i)) {
                    const Key k = key_of(v[i], (unsigned)pos(i));
                    best = k > best ? k : best;
                }
            sThread[tid] = best;
            if (tid == 0) sKey = 1;                                               // every candidate there is
            __syncthreads();
            int r = 0;
#pragma unroll 8
            for (int i = 0; i < THREADS; ++i) r += sThread[i] > best;
            if (best != 0 && r == keep - 1) sKey = best;                          // keys are unique: one thread
            if (tid == 0) sCount = held;
            __syncthreads();
            const Key from = sKey;
            if (best >= from)
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if (there(i)) {
                        const Key k = key_of(v[i], (unsigned)pos(i));
                        if (k >= from) sList[atomicAdd(&sCount, 1)] = k;          // held + keep * E at most
                    }
            __syncthreads();
            count = sCount;
        }
        if (final) {
            rank(count, out);
            for (int i = count + (int)tid; i < keep; i += THREADS) out[i] = 0;
            if (tid == THREADS - 1) {
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) s += sSum[w];
                p.sums[row * p.pieces + piece] = make_float2(m, s);
            }
        } else if (count > kList / 4) {                                           // room for the next chunk's: the best alone
            rank(count, sBest);
            __syncthreads();
            const int kept = min(count, keep);
            if (tid < (unsigned)kept) sList[tid] = sBest[tid];
            if (tid == 0) sCount = kept;
            bound = fmaxf(bound, kept == keep ? key_logit(sBest[keep - 1]) : -INFINITY);
        }
    }
}

// A workgroup per sequence.  A wave per row merges the pieces.  The largest of the lists' last logits is a bound that `keep` candidates
// reach; so is, of at least `keep` groups of lists, the least of the groups' best.  What reaches both is moved together, and its
// places are counted.  Then the rows of the sequence in the same way, by their scores: equal
// ones by their places, which are in the order of row and rank; eight lanes count a place (a lane each: 16 rows of 32 16.7 us, 11.1 with eight).
__global__ __launch_bounds__(1024) void beam_merge_kernel(const BeamParams p)
{
    constexpr int KEYS = 2;                                                       // of a lane at a time
    __shared__ __attribute__((aligned(16))) Key sLists[kMergeKeys];
    __shared__ double sScore[SSMV_BEAMS_MAX * SSMV_BEAMS_MAX];
    __shared__ int sToken[SSMV_BEAMS_MAX * SSMV_BEAMS_MAX], sDone[SSMV_BEAMS_MAX];
    __shared__ double sBound[7];
    __shared__ int sCount;
    const unsigned tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6, waves = blockDim.x >> 6;
    const int W = p.beams_in, keep = p.keep, pieces = p.pieces, n = pieces * keep;
    const size_t row0 = (size_t)blockIdx.x * W;
    Key *list = sLists + (size_t)wave * merge_room(n);
    // groups of lanes, at least `keep`, and the lists that are spread over the lanes: both powers of two
    const int groups = keep > 1 ? 1 << (32 - __builtin_clz(keep - 1)) : 1, spread = 1 << (31 - __builtin_clz(pieces));
    if (tid == 0) sCount = 0;
    for (int r = wave; r < W; r += waves) {
        const size_t row = row0 + r;
        const Key *from = p.keys + row * n;
        // all that the row needs of memory at once, also where it turns out to be finished
        const float2 part = (int)lane < pieces ? p.sums[row * pieces + lane] : make_float2(-kTop, 0.f);      // at most 64 pieces
        const Key worst = (int)lane < pieces ? from[lane * keep + keep - 1] : 0;
        Key first = 0, second = 0;                                                // the best of the lane's lists: adjacent lanes have the same or adjacent ones
        if (groups <= spread) {
            const int at = lane * spread / 64;
            first = from[at * keep];
            if (at + spread < pieces) second = from[(at + spread) * keep];
        }
        Key k[KEYS];
        auto fetch = [&](int i0) {
#pragma unroll
            for (int u = 0; u < KEYS; ++u) k[u] = i0 + u * 64 + (int)lane < n ? from[i0 + u * 64 + lane] : 0;
        };
        fetch(0);
        const int done = p.done ? p.done[row] : 0;
        float given = p.scores[row];
        given = given != given ? -INFINITY : fminf(given, kTop);
        if (lane == 0) sDone[r] = done;
        if (done != 0) {
            for (int i = lane; i < keep; i += 64) {
                sToken[r * keep + i] = p.eos;
                sScore[r * keep + i] = i == 0 ? (double)given : -INFINITY;
            }
            continue;
        }
        const float m = combine(part.x, larger);
        float bound = combine(worst ? key_logit(worst) : -INFINITY, larger);
        const float best = fmaxf(first ? key_logit(first) : -INFINITY, second ? key_logit(second) : -INFINITY);
        bound = fmaxf(bound, combine(best, [&](float a, float b, int apart) { return apart * groups < 64 ? fmaxf(a, b) : fminf(a, b); }));
        if (groups > spread) {                                                    // few lists of many keys: j of a list reach its j-th, as below (48 rows of 8 lists of 32: merge 25 -> 13 us)
            for (int j = groups / spread; j < 2 * keep; j *= 2) {
                const int at = min(j, keep), lists = (keep + at - 1) / at;
                if (lists > pieces) continue;
                const Key own = (int)lane < pieces ? from[lane * keep + at - 1] : 0;
                const float mine = own ? key_logit(own) : -INFINITY;
                int above = 0;
                for (int i = 0; i < pieces; ++i) above += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), i)) > mine;
                bound = fmaxf(bound, combine((int)lane < pieces && above < lists ? mine : INFINITY, [](float a, float b, int) { return fminf(a, b); }));
            }
        }
        const double lse = log(wave_sum64((double)part.y * (double)__builtin_amdgcn_exp2f((part.x - m) * 1.4426950408889634f)));
        int count = 0;
        for (int i0 = 0; i0 < n; i0 += 64 * KEYS) {
            if (i0 > 0) fetch(i0);
#pragma unroll
            for (int u = 0; u < KEYS; ++u) {
                const bool in = k[u] != 0 && key_logit(k[u]) >= bound;
                const unsigned long long mask = __ballot(in);
                if (in) list[count + __builtin_popcountll(mask & ((1ull << lane) - 1))] = k[u];
                count += __builtin_popcountll(mask);
            }
        }
        if (lane == 0) list[count] = 0;                                           // they are read in pairs
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");                    // the list is this wave's own
        for (int i = lane; i < count; i += 64) {
            const Key own = list[i];
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < count; j += 2) {
                const ulonglong2 two = *reinterpret_cast<const ulonglong2 *>(list + j);
                rank += (two.x > own) + (two.y > own);
            }
            if (rank < keep) {
                const float l = key_logit(own);
                sToken[r * keep + rank] = (int)key_token(own);
                sScore[r * keep + rank] = l == -INFINITY ? -INFINITY : (double)given + ((double)l - (double)m - lse);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");                    // before the next row's list
    }
    __syncthreads();
    double bound = -INFINITY;
    if (W * keep <= kFewCandidates) {
        if (keep == p.beams_out)                                                  // a vocabulary of fewer tokens: all of them
            for (int r = 0; r < W; ++r) bound = fmax(bound, sScore[r * keep + keep - 1]);
    } else {
        // j candidates of a row reach its j-th score, so `beams_out` of all rows reach the ceil(beams_out / j)-th largest of the rows' j-th
        for (int e = wave; e < 7 && 1 << e < 2 * keep; e += waves) {
            const int j = min(1 << e, keep), rows = (p.beams_out + j - 1) / j;
            const double mine = (int)lane < W ? sScore[lane * keep + j - 1] : -INFINITY;
            int above = 0;
            for (int r = 0; r < W; ++r) above += lane_get(mine, r) > mine;
            double low = (int)lane < W && above < rows ? mine : INFINITY;         // ties have as many above them
            for (int apart = 1; apart < 64; apart *= 2) low = fmin(low, __shfl_xor(low, apart));
            if (lane == 0) sBound[e] = rows <= W ? low : -INFINITY;
        }
        __syncthreads();
        for (int e = 0; e < 7 && 1 << e < 2 * keep; ++e) bound = fmax(bound, sBound[e]);
    }
    int *chosen = reinterpret_cast<int *>(sLists);                                // the lists are done with
    for (int i = tid; i < W * keep; i += blockDim.x)
        if (sScore[i] >= bound) chosen[atomicAdd(&sCount, 1)] = i;
    __syncthreads();
    const int count = sCount;
    for (int c = tid / 8; c < count; c += blockDim.x / 8) {                       // eight lanes to a candidate
        const int i = chosen[c], r = i / keep;
        const double s = sScore[i];
        int rank = 0;
#pragma unroll 2
        for (int d = tid % 8; d < count; d += 8) {
            const int j = chosen[d];
            const double o = sScore[j];
            rank += o > s || (o == s && j < i);
        }
        rank += __shfl_xor(rank, 1);
        rank += __shfl_xor(rank, 2);
        rank += __shfl_xor(rank, 4);
        if (rank < p.beams_out && tid % 8 == 0) {
            const size_t at = (size_t)blockIdx.x * p.beams_out + rank, row = row0 + r;
            p.parent[at] = (int32_t)row;
            p.token[at] = sToken[i];
            p.scores_out[at] = (float)s;
            if (p.done_out) p.done_out[at] = sDone[r] != 0 || sToken[i] == p.eos;
        }
    }
}

}  // namespace

int launch_beam_select(const BeamParams &p, hipStream_t stream)
{
    const dim3 grid((unsigned)p.pieces, (unsigned)p.batch * p.beams_in);                    // at most 65535 rows (host)
    if (p.io == SSMV_BF16) {
        if (p.small) hipLaunchKernelGGL((beam_piece_kernel<SSMV_BF16, 8>), grid, dim3(THREADS), 0, stream, p);
        else hipLaunchKernelGGL((beam_piece_kernel<SSMV_BF16, 32>), grid, dim3(THREADS), 0, stream, p);
    } else {
        if (p.small) hipLaunchKernelGGL((beam_piece_kernel<SSMV_F32, 8>), grid, dim3(THREADS), 0, stream, p);
        else hipLaunchKernelGGL((beam_piece_kernel<SSMV_F32, 32>), grid, dim3(THREADS), 0, stream, p);
    }
    const int e = (int)hipGetLastError();
    if (e != 0) return e;
    int waves = kMergeKeys / merge_room(p.pieces * p.keep);                                 // at least 3 (beam_plan)
    waves = waves < 16 ? waves : 16;
    const int wanted = p.beams_in > 4 ? p.beams_in : 4;
    hipLaunchKernelGGL(beam_merge_kernel, dim3((unsigned)p.batch), dim3(64 * (waves < wanted ? waves : wanted)), 0, stream, p);
    return (int)hipGetLastError();
}

}  // namespace ssmv
