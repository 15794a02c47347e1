// Keys and values into the 4-bit cache, and back out of it.
//
// 32 consecutive values of a head row share a scale 2^e, the least with max|x| < 7 * 2^e (so the largest is off by at
// most half a step of E2M1 plus the saturation of (6, 7) to 6), e clamped to [-125, 125]; each value is the nearest of
// +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} * 2^e, ties to the even code. A group with an infinity or a NaN has scale byte 255 and
// reads back as NaN. Scales are powers of two and every threshold is exact, so the codes do not depend on how they are
// computed; the conversion instructions (v_cvt_scalef32_pk_fp4_bf16, v_cvt_scalef32_pk_bf16_fp4) are exact here.
//
// Bound by memory: 4 D bytes of bf16 in and 17/16 D out a token and head (read: the reverse). A lane holds 8 values of
// a key row and of the value row (16 bytes each); four lanes share a scale. A work-group's lanes cover 16 tokens (D 64: of
// two heads) before the next head: nearly always a record or two, whose lines then fill in one L2 before they leave it (32,768
// tokens of 8 heads of 128, append and read: 4 / 8 / 16 / 32 tokens 78.7 / 74.8 / 71.9 / 74.3 us; with 4 the append wrote 1.4
// times its bytes). What is read goes past the L2 (non-temporal stores, 71.9 -> 62.8; of the inputs too: 61.8, but 500 tokens
// 4.95 -> 5.35). A copy of the same bytes would take 72.
#include "kv_cache.h"

namespace elis {

namespace {

constexpr int kThreads = 256;

__global__ __launch_bounds__(kWave) void kv_init_kernel(uint32_t* status) {
    if (threadIdx.x < kCacheHeader / 4) status[threadIdx.x] = 0u;
}

__device__ __forceinline__ uint32_t quad_maxu(uint32_t v) {
    uint32_t o = __shfl_xor(v, 1, kWave);
    v = v > o ? v : o;
    o = __shfl_xor(v, 2, kWave);
    return v > o ? v : o;
}

// E8M0 byte of a group whose largest magnitude has the bf16 bits `top` (sign cleared).
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    if (top >= 0x7F80u) return 255u;
    const int e = static_cast<int>(top >> 7) - 2 + ((top & 0x7Fu) >= 0x60u ? 1 : 0);  // mantissa >= 1.75
    return static_cast<uint32_t>(e < 2 ? 2 : e > 252 ? 252 : e);
}

// 8 bf16 (4 dwords) -> 8 codes in a dword.
__device__ __forceinline__ uint32_t codes_of(u32x4 x, uint32_t sb) {
#if defined(__HIP_DEVICE_COMPILE__)
    if (sb == 255u) return 0u;
    const float s = __uint_as_float(sb << 23);
    const uint32_t w0 = x[0], w1 = x[1], w2 = x[2], w3 = x[3];  // __builtin_bit_cast of a vector's element takes element 0
    uint32_t r = 0u;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w0), s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w1), s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w2), s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, w3), s, 3);
    return r;
#else
    return 0u;
#endif
}

__device__ __forceinline__ u32x4 values_of(uint32_t codes, uint32_t sb) {
    u32x4 r = {0u, 0u, 0u, 0u};
#if defined(__HIP_DEVICE_COMPILE__)
    const float s = __uint_as_float(sb << 23);
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3));
#endif
    return r;
}

__device__ __forceinline__ uint32_t top_of(u32x4 x) {
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = x[i] & 0x7FFFu, hi = (x[i] >> 16) & 0x7FFFu;
        m = m > lo ? m : lo;
        m = m > hi ? m : hi;
    }
    return m;
}

template <bool VEC>
__device__ __forceinline__ u32x4 load8(const uint16_t* p) {
    if constexpr (VEC) return *reinterpret_cast<const u32x4*>(p);
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = p[2 * i] | (static_cast<uint32_t>(p[2 * i + 1]) << 16);
    return r;
}

template <bool VEC>
__device__ __forceinline__ void store8(uint16_t* p, u32x4 x) {
    if constexpr (VEC) {
        __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(p));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[2 * i] = static_cast<uint16_t>(x[i]);
            p[2 * i + 1] = static_cast<uint16_t>(x[i] >> 16);
        }
    }
}

// Unit u of a call: lane part `sub` (8 values) of token t and head h; kKvTogether tokens are adjacent.
template <int D>
__device__ __forceinline__ void unit_of(long long u, int heads, long long* t, int* h, int* sub) {
    constexpr int L = D / 8;
    *sub = static_cast<int>(u % L);
    u /= L;
    const int b = static_cast<int>(u % kKvTogether);
    u /= kKvTogether;
    *h = static_cast<int>(u % heads);
    *t = u / heads * kKvTogether + b;
}

template <int D, bool VEC>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(KvCacheView c, const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
                                                             long long k_stride, long long v_stride, const int32_t* __restrict__ map, int n) {
    using R = Rec<D>;
    long long t;
    int h, sub;
    unit_of<D>(static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x, c.n_kv_heads, &t, &h, &sub);
    if (t >= n) return;  // the four lanes of a scale have the same t
    const int at = map[t];
    const int page = at >> c.page_shift, pos = at & (c.page_tokens - 1), tok = pos & (kRecTokens - 1);
    if (at == -1) return;  // a token without a slot
    if (at < 0 || page >= c.n_pages) {
        if (h == 0 && sub == 0) atomicOr(c.status, ELIS_DEV_BAD_PAGE);
        return;
    }
    const u32x4 xk = load8<VEC>(k + t * k_stride + h * D + 8 * sub), xv = load8<VEC>(v + t * v_stride + h * D + 8 * sub);
    const uint32_t sk = scale_byte(quad_maxu(top_of(xk))), sv = scale_byte(quad_maxu(top_of(xv)));
    const uint32_t ck = codes_of(xk, sk), cv = codes_of(xv, sv);
    uint8_t* rec = c.pages + rec_offset(c, page, h, pos / kRecTokens);
    *reinterpret_cast<uint32_t*>(rec + R::key_at(tok, 4 * sub)) = ck;
    if constexpr (D == 128) {
        *reinterpret_cast<uint32_t*>(rec + R::val_at(tok, sub)) = cv;
    } else {
        *reinterpret_cast<uint16_t*>(rec + R::val_at(tok, 2 * sub)) = static_cast<uint16_t>(cv);
        *reinterpret_cast<uint16_t*>(rec + R::val_at(tok, 2 * sub + 1)) = static_cast<uint16_t>(cv >> 16);
    }
    if ((sub & 3) == 0) {
        rec[R::scale_k_at(tok, sub / 4)] = static_cast<uint8_t>(sk);
        rec[R::scale_v_at(tok, sub / 4)] = static_cast<uint8_t>(sv);
    }
}

template <int D, bool VEC>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvCacheView c, const int32_t* __restrict__ map, int n, uint16_t* __restrict__ k,
                                                           uint16_t* __restrict__ v, long long k_stride, long long v_stride) {
    using R = Rec<D>;
    long long t;
    int h, sub;
    unit_of<D>(static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x, c.n_kv_heads, &t, &h, &sub);
    if (t >= n) return;
    const int at = map[t];
    const int page = at >> c.page_shift, pos = at & (c.page_tokens - 1), tok = pos & (kRecTokens - 1);
    u32x4 xk = {0u, 0u, 0u, 0u}, xv = xk;
    if (at >= 0 && page < c.n_pages) {
        const uint8_t* rec = c.pages + rec_offset(c, page, h, pos / kRecTokens);
        const uint32_t ck = *reinterpret_cast<const uint32_t*>(rec + R::key_at(tok, 4 * sub));
        uint32_t cv;
        if constexpr (D == 128) cv = *reinterpret_cast<const uint32_t*>(rec + R::val_at(tok, sub));
        else
            cv = *reinterpret_cast<const uint16_t*>(rec + R::val_at(tok, 2 * sub)) |
                 (static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(rec + R::val_at(tok, 2 * sub + 1))) << 16);
        xk = values_of(ck, rec[R::scale_k_at(tok, sub / 4)]);
        xv = values_of(cv, rec[R::scale_v_at(tok, sub / 4)]);
    } else if (at != -1 && h == 0 && sub == 0) {
        atomicOr(c.status, ELIS_DEV_BAD_PAGE);
    }
    store8<VEC>(k + t * k_stride + h * D + 8 * sub, xk);
    store8<VEC>(v + t * v_stride + h * D + 8 * sub, xv);
}

dim3 grid_for(const KvCacheView& c, int n) {
    const long long units = (static_cast<long long>(n) + kKvTogether - 1) / kKvTogether * kKvTogether * c.n_kv_heads * (c.d_head / 8);
    return dim3(static_cast<unsigned>((units + kThreads - 1) / kThreads));
}

bool vec_ok(const void* k, const void* v, long long k_stride, long long v_stride) {
    return ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15) == 0 && ((k_stride | v_stride) & 7) == 0;
}

}  // namespace

hipError_t launch_kv_init(KvCacheView c, hipStream_t st) {
    return launch_kernel(kv_init_kernel, dim3(1), dim3(kWave), 0, st, c.status);
}

hipError_t launch_kv_append(KvCacheView c, const uint16_t* k, const uint16_t* v, long long k_stride, long long v_stride, const int32_t* map, int n,
                            hipStream_t st) {
    const bool vec = vec_ok(k, v, k_stride, v_stride);
    const auto f = c.d_head == 128 ? (vec ? kv_append_kernel<128, true> : kv_append_kernel<128, false>)
                                   : (vec ? kv_append_kernel<64, true> : kv_append_kernel<64, false>);
    return launch_kernel(f, grid_for(c, n), dim3(kThreads), 0, st, c, k, v, k_stride, v_stride, map, n);
}

hipError_t launch_kv_read(KvCacheView c, const int32_t* map, int n, uint16_t* k, uint16_t* v, long long k_stride, long long v_stride,
                          hipStream_t st) {
    const bool vec = vec_ok(k, v, k_stride, v_stride);
    const auto f = c.d_head == 128 ? (vec ? kv_read_kernel<128, true> : kv_read_kernel<128, false>)
                                   : (vec ? kv_read_kernel<64, true> : kv_read_kernel<64, false>);
    return launch_kernel(f, grid_for(c, n), dim3(kThreads), 0, st, c, map, n, k, v, k_stride, v_stride);
}

}  // namespace elis
