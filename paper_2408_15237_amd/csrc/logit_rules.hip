// Rules on logits ahead of the choice: penalties for repeated tokens, biases, grammar masks; and the histories that the penalties count in.
#include "layers_internal.h"

namespace ssmv {
namespace {

// A token's entry: how often it was said (19 bits), whether the prompt has it, and 4095 minus the first place of it in the list of biases (0: none).
constexpr uint32_t kCount = (1u << 19) - 1, kPrompt = 1u << 19, kOccurs = kCount | kPrompt;

// A workgroup takes N tokens of a row.  It counts the row's history and enters the list of biases in a table in LDS (whole numbers, so that the order of the atomics
// does not show), then streams its logits: where the mask allows none of 8 they are not read, and in place those that nothing changes are neither read nor written.
template <int IO, int N>
__global__ __launch_bounds__(256) void logit_rules_kernel(const RulesParams p)
{
    __shared__ __attribute__((aligned(16))) uint32_t table[N];
    __shared__ int repeats;                                        // a token that is more than once in the list
    const int b = blockIdx.y, tid = (int)threadIdx.x, v0 = (int)blockIdx.x * N, n = min(N, p.V - v0);
    const bool counted = p.hist || p.bias_token;
    const int32_t *bias_token = p.bias_token ? p.bias_token + (size_t)b * p.bias_n : nullptr;
    if (counted) {
        for (int i = tid; i < N / 4; i += 256) reinterpret_cast<uint4 *>(table)[i] = make_uint4(0, 0, 0, 0);
        if (tid == 0) repeats = 0;
        __syncthreads();
        if (bias_token) {
            for (int j = tid; j < p.bias_n; j += 256) {
                const unsigned at = (unsigned)bias_token[j] - (unsigned)v0;           // negative tokens: far beyond n
                if (at < (unsigned)n) atomicMax(&table[at], (uint32_t)(4095 - j) << 20);
            }
            __syncthreads();
            for (int j = tid; j < p.bias_n; j += 256) {
                const unsigned at = (unsigned)bias_token[j] - (unsigned)v0;
                if (at < (unsigned)n && table[at] >> 20 != (uint32_t)(4095 - j)) repeats = 1;
            }
            __syncthreads();
        }
        if (p.hist) {
            const int src = p.src_row ? p.src_row[b] : b;
            const bool have = (unsigned)src < (unsigned)p.rows_in;
            const int len = have ? min(max(p.hist_len[src], 0), p.room) : 0, prompt = p.prompt_len ? p.prompt_len[b] : 0;
            const int32_t *hist = p.hist + (size_t)(have ? src : 0) * p.room;
            int32_t *to = blockIdx.x == 0 && p.hist_out ? p.hist_out + (size_t)b * p.room : nullptr;
            auto count = [&](int token, int t) {
                const unsigned at = (unsigned)token - (unsigned)v0;
                if (at >= (unsigned)n) return;
                if (t < prompt) atomicOr(&table[at], kPrompt);
                else atomicAdd(&table[at], 1u);
            };
            for (int t = tid; t < len; t += 256) {
                const int token = hist[t];
                count(token, t);
                if (to && to != hist) to[t] = token;
            }
            if (tid == 0 && p.token) {
                count(p.token[b], len);
                if (to && len < p.room) to[len] = p.token[b];
            }
            if (tid == 0 && to) p.hist_len_out[b] = min(len + (p.token ? 1 : 0), p.room);
        }
        __syncthreads();
    }
    const float rep = p.repetition ? p.repetition[b] : 1.f, freq = p.frequency ? p.frequency[b] : 0.f, pres = p.presence ? p.presence[b] : 0.f;
    const int mrow = p.mask ? (p.mask_row ? p.mask_row[b] : b) : -1;
    const unsigned char *mask = p.mask && (unsigned)mrow < (unsigned)p.mask_rows ? reinterpret_cast<const unsigned char *>(p.mask + (size_t)mrow * p.mask_stride) : nullptr;
    const bool in_place = p.out == p.logits;
    auto edit = [&](float l, uint32_t e) {
        if (e & kOccurs) {
            l = l > 0.f ? l / rep : l * rep;
            if (e & kCount) l = l - freq * (float)(e & kCount) - pres;
        }
        if (e >> 20) {
            const int j = 4095 - (int)(e >> 20);
            float s = p.bias[(size_t)b * p.bias_n + j];
            if (repeats) {
                const int token = bias_token[j];
                for (int i = j + 1; i < p.bias_n; ++i)
                    if (bias_token[i] == token) s += p.bias[(size_t)b * p.bias_n + i];
            }
            l += s;
        }
        return l;
    };
    for (int at = tid * 8; at < n; at += 256 * 8) {
        const int v = v0 + at, live = min(n - at, 8);
        const unsigned char bits = mask ? mask[v / 8] : 0xff;
        uint32_t e[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (counted) {
            const uint4 lo = *reinterpret_cast<const uint4 *>(table + at), hi = *reinterpret_cast<const uint4 *>(table + at + 4);
            e[0] = lo.x; e[1] = lo.y; e[2] = lo.z; e[3] = lo.w; e[4] = hi.x; e[5] = hi.y; e[6] = hi.z; e[7] = hi.w;
        }
        const uint32_t any = e[0] | e[1] | e[2] | e[3] | e[4] | e[5] | e[6] | e[7];
        if (in_place && any == 0 && bits == 0xff) continue;
        float l[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) l[j] = 0.f;
        if (bits != 0) load8<IO>(p.logits, (size_t)b * p.row_stride + v, live, l);
        if (any != 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (e[j] != 0) l[j] = edit(l[j], e[j]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) l[j] = bits >> j & 1 ? l[j] : -__builtin_inff();
        store8<IO>(p.out, (size_t)b * p.out_stride + v, live, l);
    }
}

template <int IO>
int launch(const RulesParams &p, hipStream_t stream)
{
    if ((size_t)p.rows * ((p.V + 8191) / 8192) >= 512) hipLaunchKernelGGL((logit_rules_kernel<IO, 8192>), dim3((p.V + 8191) / 8192, p.rows), dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((logit_rules_kernel<IO, 2048>), dim3((p.V + 2047) / 2048, p.rows), dim3(256), 0, stream, p);
    return (int)hipGetLastError();
}

}  // namespace

int launch_logit_rules(const RulesParams &p, hipStream_t stream)
{
    return p.io == SSMV_BF16 ? launch<SSMV_BF16>(p, stream) : launch<SSMV_F32>(p, stream);
}

}  // namespace ssmv
