// Penalties for repeated tokens, biases and grammar masks on the next token's logits.
//
// For row i and token v, with h = v occurs in the row's history and c = its occurrences past the prompt:
//   y = h ? (x > 0 ? x / r : x * r) : x,  y -= f * c,  y -= p if c > 0,  y += sum of v's biases,  -inf if v's mask bit is 0
// all in fp32. The logits are read once and written once; everything else is small beside them. A work-group takes a
// row's stretch of kChunk tokens, counts the history's tokens that fall into it in LDS (every work-group of a row
// reads the whole history, which the L2 holds), and then passes over the stretch. A row's few biases are added at the
// end by one thread each; of a token named more than once the first entry adds them all, in list order, so the result
// does not depend on timing. The counters are integers: the order of their atomics does not matter either.
#include <math.h>

#include "kernels.h"

namespace elis {

namespace {

constexpr int kThreads = 512;
constexpr int kChunk = 8192;          // tokens of a work-group
constexpr uint32_t kPrompt = 1u << 31;  // seen in the prompt; below it the count past the prompt

template <bool BF16>
__device__ __forceinline__ float load1(const void* p, long long i) {
    if constexpr (BF16) return bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
    return static_cast<const float*>(p)[i];
}

template <bool BF16>
__device__ __forceinline__ f32x4 load4(const void* p, long long i, bool vec) {
    if (!vec) return f32x4{load1<BF16>(p, i), load1<BF16>(p, i + 1), load1<BF16>(p, i + 2), load1<BF16>(p, i + 3)};
    if constexpr (BF16) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(p) + i);
        return f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xFFFF0000u), __uint_as_float(w[1] << 16),
                     __uint_as_float(w[1] & 0xFFFF0000u)};
    }
    return *reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + i);
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void logits_adjust_kernel(LogitsArgs a) {
    __shared__ __attribute__((aligned(16))) uint32_t seen[kChunk + 4];
    const int row = blockIdx.y, tid = threadIdx.x;
    const float* out_row0 = a.out + static_cast<long long>(row) * a.out_stride;
    float* out = a.out + static_cast<long long>(row) * a.out_stride;
    const void* in = BF16 ? static_cast<const void*>(static_cast<const uint16_t*>(a.logits) + static_cast<long long>(row) * a.in_stride)
                          : static_cast<const void*>(static_cast<const float*>(a.logits) + static_cast<long long>(row) * a.in_stride);
    // Stretches start where the output is 16-byte aligned; the first one takes the up to three tokens before that too.
    const int lead = static_cast<int>((0 - (reinterpret_cast<uintptr_t>(out_row0) >> 2)) & 3);
    const int body = lead + blockIdx.x * kChunk;
    if (blockIdx.x > 0 && body >= a.vocab) return;
    const int v0 = blockIdx.x == 0 ? 0 : body, skip = body - v0;
    const int v1 = body + kChunk < a.vocab ? body + kChunk : a.vocab;

    for (int i = tid; i < (kChunk + 4) / 4; i += kThreads) reinterpret_cast<u32x4*>(seen)[i] = u32x4{0u, 0u, 0u, 0u};
    const float rep = a.repetition ? a.repetition[row] : 1.0f, freq = a.frequency ? a.frequency[row] : 0.0f,
                pres = a.presence ? a.presence[row] : 0.0f;
    __syncthreads();
    if (a.token_ids) {
        long long t0 = a.cu[row], t1 = a.cu[row + 1];
        t0 = t0 < 0 ? 0 : t0;
        t1 = t1 < a.total_tokens ? t1 : a.total_tokens;
        const long long prompt = t0 + (a.prompt_lens ? a.prompt_lens[row] : 0);
        for (long long t = t0 + tid; t < t1; t += kThreads) {
            const long long at = static_cast<long long>(a.token_ids[t]) - v0;
            if (at >= 0 && at < v1 - v0) {
                // counter of token v0 + at; the body's are 16-byte aligned at seen[4]
                uint32_t* s = &seen[at - skip + 4];
                if (t < prompt) atomicOr(s, kPrompt);
                else atomicAdd(s, 1u);
            }
        }
        __syncthreads();
    }
    const int32_t mask_row = a.mask && a.mask_rows ? a.mask_rows[row] : a.mask ? row : -1;
    const uint32_t* mask = mask_row >= 0 && mask_row < a.n_masks ? a.mask + static_cast<long long>(mask_row) * a.mask_stride : nullptr;

    auto adjust = [&](float x, uint32_t s) {
        if (s == 0u) return x;
        x = x > 0.f ? x / rep : x * rep;
        const uint32_t c = s & ~kPrompt;
        if (c) x = __fsub_rn(__fsub_rn(x, __fmul_rn(freq, static_cast<float>(c))), pres);
        return x;
    };
    if (tid < skip && tid < v1) {
        float y = adjust(load1<BF16>(in, tid), seen[tid - skip + 4]);
        if (mask && !((mask[tid >> 5] >> (tid & 31)) & 1u)) y = -INFINITY;
        out[tid] = y;
    }
    const bool vec = BF16 ? ((reinterpret_cast<uintptr_t>(in) + 2 * static_cast<uintptr_t>(body)) & 7) == 0
                          : ((reinterpret_cast<uintptr_t>(in) + 4 * static_cast<uintptr_t>(body)) & 15) == 0;
    for (int v = body + 4 * tid; v < v1; v += 4 * kThreads) {
        const u32x4 s = *reinterpret_cast<const u32x4*>(&seen[v - body + 4]);
        if (v + 4 <= v1) {
            f32x4 x = load4<BF16>(in, v, vec);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = adjust(x[e], s[e]);
            if (mask) {
                const uint32_t lo = mask[v >> 5], hi = mask[(v + 3) >> 5];
                const uint32_t bits = static_cast<uint32_t>((static_cast<uint64_t>(hi) << 32 | lo) >> (v & 31));
                // with all four in one word hi equals lo and its copy lies past them
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!((bits >> e) & 1u)) x[e] = -INFINITY;
            }
            *reinterpret_cast<f32x4*>(out + v) = x;
        } else {
            for (int e = 0; v + e < v1; ++e) {
                float y = adjust(load1<BF16>(in, v + e), s[e]);
                if (mask && !((mask[(v + e) >> 5] >> ((v + e) & 31)) & 1u)) y = -INFINITY;
                out[v + e] = y;
            }
        }
    }
    if (a.bias_cu) {
        long long b0 = a.bias_cu[row], b1 = a.bias_cu[row + 1];
        b0 = b0 < 0 ? 0 : b0;
        b1 = b1 < a.bias_total ? b1 : a.bias_total;
        if (b0 >= b1) return;
        __syncthreads();  // the stretch is written
        for (long long i = b0 + tid; i < b1; i += kThreads) {
            const int v = a.bias_tokens[i];
            if (v < v0 || v >= v1) continue;
            bool first = true;
            for (long long j = b0; j < i && first; ++j) first = a.bias_tokens[j] != v;
            if (!first) continue;
            float sum = a.bias_values[i];
            for (long long j = i + 1; j < b1; ++j)
                if (a.bias_tokens[j] == v) sum += a.bias_values[j];
            if (!mask || ((mask[v >> 5] >> (v & 31)) & 1u)) out[v] += sum;
        }
    }
}

}  // namespace

hipError_t launch_logits_adjust(const LogitsArgs& a, hipStream_t st) {
    const dim3 grid(static_cast<unsigned>((a.vocab + kChunk - 1) / kChunk), static_cast<unsigned>(a.n));
    return a.bf16 ? launch_kernel(logits_adjust_kernel<true>, grid, dim3(kThreads), 0, st, a)
                  : launch_kernel(logits_adjust_kernel<false>, grid, dim3(kThreads), 0, st, a);
}

}  // namespace elis
