// Penalties for repeated tokens, biases and grammar masks on the next token's logits.
//
// For row i and token v, with h = v occurs in the row's history and c = its occurrences past the prompt:
//   y = h ? (x > 0 ? x / r : x * r) : x,  y -= f * c,  y -= p if c > 0,  y += sum of v's biases,  -inf if v's mask bit is 0
// all in fp32. The logits are read once and written once; everything else is small beside them. A work-group takes a
// row's stretch of kChunk tokens: it requests the stretch's logits, counts the history's tokens that fall into it in LDS
// (every work-group of a row reads the whole history, which the L2 holds), sums the row's biases of its tokens into LDS,
// and then makes one pass over the registers. Biases of one token are added up in list order, so the result does not
// depend on timing; the counters are integers, whose atomics commute.
#include <math.h>

#include "kernels.h"

namespace elis {

namespace {

// 128 rows of 250,002 fp32 logits, 32 of 30,522 bf16: 512 threads and 4,096 tokens 62 / 5.9 us, 512 and 8,192 70 / 7.1,
// 1,024 and 8,192 60 / 6.4, 256 and 4,096 78 / 7.5, 512 and 2,048 88 / 5.9 (without the early loads, and with the biases
// added to the written output, 105 / 8.5). Loads and stores past the
// L2, since nothing here is read again, 57.5 / 6.0 (only the stores 62 / 5.9, neither 69.6 / 5.9): 4.5 TB/s; a copy of 4 GiB runs at 4.7.
constexpr int kThreads = 512;
constexpr int kChunk = 4096;          // tokens of a work-group
constexpr int kVecs = kChunk / (4 * kThreads);  // groups of four a thread
constexpr uint32_t kPrompt = 1u << 31;  // seen in the prompt
constexpr uint32_t kBias = 1u << 30;    // has a bias; below it the count past the prompt
constexpr int kTurns = 1024;            // places at which the entries of a bias list take turns

template <bool BF16>
__device__ __forceinline__ float load1(const void* p, long long i) {
    if constexpr (BF16) return bf16_to_f32(static_cast<const uint16_t*>(p)[i]);
    return static_cast<const float*>(p)[i];
}

template <bool BF16>
__device__ __forceinline__ f32x4 load4(const void* p, long long i) {
    if constexpr (BF16) {
        const u32x2 w = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(p) + i));
        return f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xFFFF0000u), __uint_as_float(w[1] << 16),
                     __uint_as_float(w[1] & 0xFFFF0000u)};
    }
    return __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + i));
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void logits_adjust_kernel(LogitsArgs a) {
    __shared__ __attribute__((aligned(16))) uint32_t seen[kChunk + 4];
    __shared__ float bias[kChunk + 4];  // of the tokens whose counter has kBias
    __shared__ int turn[kTurns];
    const int row = blockIdx.y, tid = threadIdx.x;
    float* out = a.out + static_cast<long long>(row) * a.out_stride;
    const void* in = BF16 ? static_cast<const void*>(static_cast<const uint16_t*>(a.logits) + static_cast<long long>(row) * a.in_stride)
                          : static_cast<const void*>(static_cast<const float*>(a.logits) + static_cast<long long>(row) * a.in_stride);
    // Stretches start where the output is 16-byte aligned; the first one takes the up to three tokens before that too.
    const int lead = static_cast<int>((0 - (reinterpret_cast<uintptr_t>(out) >> 2)) & 3);
    const int body = lead + blockIdx.x * kChunk;
    if (blockIdx.x > 0 && body >= a.vocab) return;
    const int v0 = blockIdx.x == 0 ? 0 : body, skip = body - v0;
    const int v1 = body + kChunk < a.vocab ? body + kChunk : a.vocab;

    const float rep = a.repetition ? a.repetition[row] : 1.0f, freq = a.frequency ? a.frequency[row] : 0.0f,
                pres = a.presence ? a.presence[row] : 0.0f;
    const int32_t mask_row = a.mask && a.mask_rows ? a.mask_rows[row] : a.mask ? row : -1;
    const uint32_t* mask = mask_row >= 0 && mask_row < a.n_masks ? a.mask + static_cast<long long>(mask_row) * a.mask_stride : nullptr;
    long long t0 = 0, t1 = 0, prompt = 0, b0 = 0, b1 = 0;
    if (a.token_ids) {
        t0 = a.cu[row];
        t1 = a.cu[row + 1];
        t0 = t0 < 0 ? 0 : t0;
        t1 = t1 < a.total_tokens ? t1 : a.total_tokens;
        prompt = t0 + (a.prompt_lens ? a.prompt_lens[row] : 0);
    }
    if (a.bias_cu) {
        b0 = a.bias_cu[row];
        b1 = a.bias_cu[row + 1];
        b0 = b0 < 0 ? 0 : b0;
        b1 = b1 < a.bias_total ? b1 : a.bias_total;
    }

    // The stretch's logits are requested first: they arrive while the history is counted.
    const bool vec = BF16 ? ((reinterpret_cast<uintptr_t>(in) + 2 * static_cast<uintptr_t>(body)) & 7) == 0
                          : ((reinterpret_cast<uintptr_t>(in) + 4 * static_cast<uintptr_t>(body)) & 15) == 0;
    f32x4 x[kVecs];
    if (vec && body + kChunk <= a.vocab) {  // uniform
#pragma unroll
        for (int y = 0; y < kVecs; ++y) x[y] = load4<BF16>(in, body + 4 * (tid + y * kThreads));
    } else {
#pragma unroll
        for (int y = 0; y < kVecs; ++y) {
            const int v = body + 4 * (tid + y * kThreads);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[y][e] = v + e < v1 ? load1<BF16>(in, v + e) : 0.f;
        }
    }
    // Bit 4 y + e: the mask forbids element e of group y.
    uint32_t forbid = 0u;
    if (mask) {
#pragma unroll
        for (int y = 0; y < kVecs; ++y) {
            const int v = body + 4 * (tid + y * kThreads), last = v + 3 < v1 ? v + 3 : v1 - 1;
            if (v < v1) {
                const uint32_t lo = mask[v >> 5], hi = mask[last >> 5];  // in one word: hi equals lo and lies past the four
                forbid |= (~static_cast<uint32_t>((static_cast<uint64_t>(hi) << 32 | lo) >> (v & 31)) & 15u) << (4 * y);
            }
        }
    }

    for (int i = tid; i < (kChunk + 4) / 4; i += kThreads) reinterpret_cast<u32x4*>(seen)[i] = u32x4{0u, 0u, 0u, 0u};
    __syncthreads();
    // Counter of token v0 + at: the body's are 16-byte aligned at seen[4].
    for (long long base = t0; base < t1; base += 4 * kThreads) {
        int32_t id[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const long long t = base + tid + y * kThreads;
            id[y] = t < t1 ? a.token_ids[t] : -1;
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const long long at = static_cast<long long>(id[y]) - v0;
            if (at >= 0 && at < v1 - v0) {
                uint32_t* s = &seen[at - skip + 4];
                if (base + tid + y * kThreads < prompt) atomicOr(s, kPrompt);
                else atomicAdd(s, 1u);
            }
        }
    }
    // Biases, an entry a thread and kThreads of the list at a time. Entries whose tokens share a place of `turn` (those of
    // one token do) go one after the other in list order; nearly always there is one turn. A work-group none of whose
    // tokens the entries name passes one barrier.
    if (b0 < b1) {
        for (int i = tid; i < kTurns; i += kThreads) turn[i] = kThreads;
        for (long long base = b0; base < b1; base += kThreads) {
            const long long i = base + tid;
            const int v = i < b1 ? a.bias_tokens[i] : -1;
            bool waits = v >= v0 && v < v1;
            const int at = v - body + 4;
            const float add = waits ? a.bias_values[i] : 0.f;
            while (__syncthreads_or(waits)) {
                int* place = &turn[at & (kTurns - 1)];
                if (waits) atomicMin(place, tid);
                __syncthreads();
                const bool mine = waits && *place == tid;
                if (mine) {
                    const uint32_t s = seen[at];
                    bias[at] = s & kBias ? bias[at] + add : add;
                    seen[at] = s | kBias;
                    waits = false;
                }
                __syncthreads();
                if (mine) *place = kThreads;
            }
        }
    }
    __syncthreads();

    auto adjust = [&](float z, uint32_t s, int at) {
        if (s & ~kBias) z = z > 0.f ? z / rep : z * rep;
        const uint32_t c = s & ~(kPrompt | kBias);
        if (c) z = __fsub_rn(__fsub_rn(z, __fmul_rn(freq, static_cast<float>(c))), pres);
        if (s & kBias) z += bias[at];
        return z;
    };
    if (tid < skip && tid < v1) {
        const int at = tid - skip + 4;
        float z = adjust(load1<BF16>(in, tid), seen[at], at);
        if (mask && !((mask[tid >> 5] >> (tid & 31)) & 1u)) z = -INFINITY;
        out[tid] = z;
    }
#pragma unroll
    for (int y = 0; y < kVecs; ++y) {
        const int at = 4 + 4 * (tid + y * kThreads), v = body - 4 + at;
        if (v >= v1) break;
        const u32x4 s = *reinterpret_cast<const u32x4*>(&seen[at]);
        if ((s[0] | s[1] | s[2] | s[3]) != 0u) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (s[e]) x[y][e] = adjust(x[y][e], s[e], at + e);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if ((forbid >> (4 * y + e)) & 1u) x[y][e] = -INFINITY;
        if (v + 4 <= v1) {
            __builtin_nontemporal_store(x[y], reinterpret_cast<f32x4*>(out + v));
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (v + e < v1) out[v + e] = x[y][e];
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
