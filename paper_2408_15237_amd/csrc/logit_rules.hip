// Rules on logits ahead of the choice: penalties for repeated tokens, biases, grammar masks; and the histories that the penalties count in.
#include "layers_internal.h"

namespace ssmv {
namespace {

// A token's entry: how often it was said (19 bits), whether the prompt has it, and 4095 minus the first place of it in the list of biases (0: none).
constexpr uint32_t kCount = (1u << 19) - 1, kPrompt = 1u << 19, kOccurs = kCount | kPrompt;

// A workgroup takes N tokens of a row.  It counts the row's history and enters the list of biases in a table in LDS (whole numbers, so that the order of the atomics
// does not show) and then applies both to its logits: where the mask allows none of 8 they are not read, and in place those that nothing changes are neither read nor written.
// A row costs little more than its bytes, and the way to them is a chain of dependent loads (the parent's index, its length, its tokens; the mask's row, its bits, the logits):
// everything is requested as soon as its address is known, the logits before the table is built.  128 rows x 128011 bf16 out of place, us: grammars alone 13.5 (66 MB, 5 TB/s), histories of up to
// 1000 tokens 22, both and 100 biases 16 to 19 (45 with the loads where they are used, when the rest took 23); tables of 8192 tokens 31, of 2048 27; workgroups that take several pieces and ask for the next one's
// logits ahead, of which five run on a compute unit, 26.  In place, grammars alone, 64 x 49999: 5.
template <int IO, int N>
__global__ __launch_bounds__(256) void logit_rules_kernel(const RulesParams p)
{
    constexpr int V8 = N / 8 / 256, H = 4;                          // vectors of 8 tokens a thread; tokens of the history that it asks for ahead
    __shared__ __attribute__((aligned(16))) uint32_t table[N];
    __shared__ int repeats;                                        // a token that is more than once in the list
    extern __shared__ float bias_of[];                             // [bias_n]
    const int b = blockIdx.y, tid = (int)threadIdx.x, v0 = (int)blockIdx.x * N, n = min(N, p.V - v0);
    const bool counted = p.hist || p.bias_token, in_place = p.out == p.logits;
    const int32_t *bias_token = p.bias_token ? p.bias_token + (size_t)b * p.bias_n : nullptr;
    const int src = p.src_row ? p.src_row[b] : b, mrow = p.mask ? (p.mask_row ? p.mask_row[b] : b) : -1;
    const int added = p.token ? p.token[b] : -1, prompt = p.prompt_len ? p.prompt_len[b] : 0;
    const float rep = p.repetition ? p.repetition[b] : 1.f, freq = p.frequency ? p.frequency[b] : 0.f, pres = p.presence ? p.presence[b] : 0.f;
    const bool known = p.hist && (unsigned)src < (unsigned)p.rows_in;
    const int32_t *hist = p.hist + (size_t)(known ? src : 0) * p.room;
    const int said = known ? p.hist_len[src] : 0;
    int32_t ahead[H];
#pragma unroll
    for (int k = 0; k < H; ++k) ahead[k] = known && tid + k * 256 < p.room ? hist[tid + k * 256] : -1;       // some of it may lie behind the history
    const bool listed = bias_token && tid < p.bias_n;
    const int list0 = listed ? bias_token[tid] : -1;
    const float bias0 = listed ? p.bias[(size_t)b * p.bias_n + tid] : 0.f;
    const unsigned char *mask = (unsigned)mrow < (unsigned)p.mask_rows && p.mask ? reinterpret_cast<const unsigned char *>(p.mask + (size_t)mrow * p.mask_stride) : nullptr;
    uint32_t bits[V8];
#pragma unroll
    for (int k = 0; k < V8; ++k) {
        const int at = (k * 256 + tid) * 8;
        bits[k] = mask && at < n ? mask[(v0 + at) / 8] : 0xffu;
    }
    float l[V8][8];
    auto fetch = [&](int k) {
        const int at = (k * 256 + tid) * 8;
        load8<IO>(p.logits, (size_t)b * p.row_stride + v0 + at, min(n - at, 8), l[k]);
    };
    if (!in_place) {
#pragma unroll
        for (int k = 0; k < V8; ++k)
            if ((k * 256 + tid) * 8 < n && bits[k] != 0) fetch(k);
    }
    if (counted) {
        for (int i = tid; i < N / 4; i += 256) reinterpret_cast<uint4 *>(table)[i] = make_uint4(0, 0, 0, 0);
        if (tid == 0) repeats = 0;
        __syncthreads();
        if (bias_token) {
            auto enter = [&](int token, float bias, int j) {
                const unsigned at = (unsigned)token - (unsigned)v0;                  // negative tokens: far beyond n
                if (at >= (unsigned)n) return;
                if (atomicMax(&table[at], (uint32_t)(4095 - j) << 20) != 0) repeats = 1;
                bias_of[j] = bias;
            };
            enter(list0, bias0, tid);
            for (int j = tid + 256; j < p.bias_n; j += 256) enter(bias_token[j], p.bias[(size_t)b * p.bias_n + j], j);
            __syncthreads();
            // What is listed again is added to its token's first place, in the order of the list: every fourth token by one wave, whose first lane holds the sum while the token stays the same.
            // 128 rows x 128011 bf16, 4095 tokens of one piece of the vocabulary, one of them twice: 118 us, 55 without (57 ms where every token of such a list looked for itself in the rest of it).
            if (__builtin_expect(repeats, 0)) {
                const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
                int first = -1;
                float sum = 0.f;
                for (int j0 = 0; j0 < p.bias_n; j0 += 64) {
                    const int j = j0 + lane;
                    const unsigned at = j < p.bias_n ? (unsigned)bias_token[j] - (unsigned)v0 : ~0u;
                    const bool mine = at < (unsigned)n && (int)(at & 3u) == wave;
                    const int to = mine ? 4095 - (int)(__hip_atomic_load(&table[at], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) >> 20) : j;      // others count by now
                    const float more = mine ? bias_of[j] : 0.f;
                    for (uint64_t again = __ballot(to != j); again != 0; again &= again - 1) {
                        const int k = __builtin_ctzll(again), next = __builtin_amdgcn_readlane(to, k);
                        if (next != first) {
                            if (first >= 0 && lane == 0) bias_of[first] = sum;
                            first = next;
                            sum = bias_of[first];
                        }
                        sum += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(more), k));
                    }
                }
                if (first >= 0 && lane == 0) bias_of[first] = sum;
            }
        }
        if (p.hist) {
            const int len = min(max(said, 0), p.room);
            int32_t *to = blockIdx.x == 0 && p.hist_out ? p.hist_out + (size_t)b * p.room : nullptr;
            auto count = [&](int token, int t) {
                const unsigned at = (unsigned)token - (unsigned)v0;
                if (at >= (unsigned)n) return;
                if (t < prompt) atomicOr(&table[at], kPrompt);
                else atomicAdd(&table[at], 1u);
            };
            auto one = [&](int token, int t) {
                if (t >= len) return;
                count(token, t);
                if (to && to != hist) to[t] = token;
            };
#pragma unroll
            for (int k = 0; k < H; ++k) one(ahead[k], tid + k * 256);
            for (int t = tid + H * 256; t < len; t += 256) one(hist[t], t);
            if (tid == 0 && p.token) {
                count(added, len);
                if (to && len < p.room) to[len] = added;
            }
            if (tid == 0 && to) p.hist_len_out[b] = min(len + (p.token ? 1 : 0), p.room);
        }
        __syncthreads();
    }
    // A read of LDS by every wave between its loads and its stores, for nothing but its time (without it grammars alone take 14.2 us for 13.5, histories 22.4 for 22.0).
    asm volatile("" ::"v"(repeats));
    auto edit = [&](float v, uint32_t e) {
        if (e & kOccurs) {
            v = v > 0.f ? v / rep : v * rep;
            if (e & kCount) v = v - freq * (float)(e & kCount) - pres;
        }
        if (e >> 20) v += bias_of[4095 - (int)(e >> 20)];
        return v;
    };
#pragma unroll
    for (int k = 0; k < V8; ++k) {
        const int at = (k * 256 + tid) * 8;
        if (at >= n) continue;
        uint32_t e[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (counted) {
            const uint4 lo = *reinterpret_cast<const uint4 *>(table + at), hi = *reinterpret_cast<const uint4 *>(table + at + 4);
            e[0] = lo.x; e[1] = lo.y; e[2] = lo.z; e[3] = lo.w; e[4] = hi.x; e[5] = hi.y; e[6] = hi.z; e[7] = hi.w;
        }
        const uint32_t any = e[0] | e[1] | e[2] | e[3] | e[4] | e[5] | e[6] | e[7];
        if (in_place) {
            if (any == 0 && bits[k] == 0xff) continue;
            if (bits[k] != 0) fetch(k);
        }
        if (any != 0 && bits[k] != 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (e[j] != 0) l[k][j] = edit(l[k][j], e[j]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) l[k][j] = bits[k] >> j & 1 ? l[k][j] : -__builtin_inff();
        store8<IO>(p.out, (size_t)b * p.out_stride + v0 + at, min(n - at, 8), l[k]);
    }
}

template <int IO>
int launch(const RulesParams &p, hipStream_t stream)
{
    const size_t lds = p.bias_token ? (size_t)p.bias_n * sizeof(float) : 0;
    auto go = [&](auto kernel, int N) { hipLaunchKernelGGL(kernel, dim3((p.V + N - 1) / N, p.rows), dim3(256), lds, stream, p); };
    // eight workgroups with a table of 4096 run on a compute unit
    if ((size_t)p.rows * ((p.V + 4095) / 4096) >= 1024) go(logit_rules_kernel<IO, 4096>, 4096);
    else go(logit_rules_kernel<IO, 2048>, 2048);
    return (int)hipGetLastError();
}

}  // namespace

int launch_logit_rules(const RulesParams &p, hipStream_t stream)
{
    return p.io == SSMV_BF16 ? launch<SSMV_BF16>(p, stream) : launch<SSMV_F32>(p, stream);
}

}  // namespace ssmv
