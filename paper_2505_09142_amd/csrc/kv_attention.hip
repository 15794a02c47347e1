// Attention of new tokens over the 4-bit paged cache.
//
// Rows. The queries of one request that read the same kv head (its new tokens times the n_heads / n_kv_heads query
// heads of the group) are the rows of one product: row r is token r / G, head r % G of the group. A work-group takes 16
// NB rows of a (request, kv head) and one chunk of the keys they see; its four waves split the chunk's keys and each
// streams its own records straight from memory into registers, so nothing but the final merge passes through LDS.
//
// Products. As the encoder's attention: S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_16x16x32_bf16, the accumulators of
// the first being, rounded to bf16, the P^T operand of the second (lane group g holds keys 4g..4g+3 of each of a step's
// two records). The order of d inside the first product and of the rows of V^T is free, so each lane takes the 16
// consecutive bytes of a record that make its operands: of the keys D/4 consecutive values of one key (within one
// scale), of the values D/16 columns of four keys. E2M1 times a power of two is exact in bf16: one
// v_cvt_scalef32_pk_bf16_fp4 makes two operands' worth, for V^T followed by one byte permutation that pairs two keys.
//
// Softmax: running maximum and sum in fp32; the maximum lags (the accumulators are rescaled only when a score exceeds
// it by 2^8), the row sum comes from the matrix cores over the bf16 weights that multiply V.
//
// Masks. A key is seen when it is at or before the token's position, inside its window, and on a valid page. Records
// wholly seen by every row skip the test. The codes of keys that no row may see (past the end, on a bad page) are
// zeroed, so what lies there cannot matter; a group of values that holds NaN (scale 255) is multiplied as zero and
// makes NaN of exactly the rows that see it.
//
// Bound by memory for single tokens: 17/16 D bytes a key and kv head, once. The vector unit comes second: about 180
// instructions a 32-key step of a wave. Few rows are split over the keys (chunks) and joined by a second launch.
#include <math.h>

#include "kv_cache.h"

namespace elis {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kStep = 32;  // keys a wave takes at a time: two records

__device__ __forceinline__ float quad_max(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

template <int D>
struct RecRegs;
template <>
struct RecRegs<128> {
    typedef u32x4 vec;
};
template <>
struct RecRegs<64> {
    typedef u32x2 vec;
};

struct Request {
    int q0, ql, kv;
    bool ok;
};

// Request i, checked against what the host was told; ok = false leaves it alone (and flags it).
__device__ __forceinline__ Request request_of(const KvAttnArgs& a, int i) {
    Request r;
    r.q0 = a.cu[i];
    const int o1 = a.cu[i + 1];
    r.ql = o1 - r.q0;
    r.kv = a.kv_lens[i];
    const bool bad_cu = r.q0 < 0 || o1 > a.total_q || o1 < r.q0;
    const bool too_long = r.ql > a.max_q || r.kv > a.max_kv || r.kv < 0;
    r.ok = !bad_cu && !too_long;
    if (!r.ok && threadIdx.x == 0) atomicOr(a.c.status, bad_cu ? ELIS_DEV_BAD_CU : ELIS_DEV_LONG_SEQ);
    return r;
}

// Keys that rows [r0, r1) of a request may see: [lo, hi), lo on a record; empty as 0, 0.
__device__ __forceinline__ void span_of(const KvAttnArgs& a, const Request& q, int r0, int r1, int* lo, int* hi) {
    const int back = q.kv - q.ql;
    const int first = back + r0 / a.group, last = back + (r1 - 1) / a.group;
    int l = a.window > 0 ? first - a.window + 1 : 0;
    l = l > 0 ? l & ~(kRecTokens - 1) : 0;
    const int h = last + 1;
    if (h <= l) {
        *lo = *hi = 0;
    } else {
        *lo = l;
        *hi = h;
    }
}

__device__ __forceinline__ int chunks_of(int lo, int hi, int chunk) {
    const int n = (hi - lo + chunk - 1) / chunk;
    return n < 1 ? 1 : n;
}

__device__ __forceinline__ float scale_of(uint32_t dword, int byte) {
    return __uint_as_float(((dword >> (8 * byte)) & 0xFFu) << 23);
}

// Four waves. MANY: rows of every request with more than `small` rows, in tiles; else the others, one tile each.
template <int D, int NB, bool MANY>
__global__ __launch_bounds__(kThreads) void kv_attention_kernel(KvAttnArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    using R = Rec<D>;
    typedef typename RecRegs<D>::vec vec;
    constexpr int KS = D / 32;   // k-steps of the first product
    constexpr int DB = D / 16;   // 16-row blocks of O^T; values of a column
    constexpr int CV = D / 64;   // conversions of a column: pairs of values
    constexpr int CVN = DB / 2;  // = 4 (D 128), 2 (D 64)
    static_assert(CVN == 2 * CV, "pairs of a column");
    __shared__ __attribute__((aligned(16))) float so[kWaves][16][D + 4];
    __shared__ float sm[kWaves][NB * 16], sl[kWaves][NB * 16];

    const int chunk_i = blockIdx.x % a.nchunks, rt = blockIdx.x / a.nchunks, h = blockIdx.y, req = blockIdx.z;
    const Request rq = request_of(a, req);
    const int rows = rq.ql * a.group;
    if (!rq.ok || rows <= 0 || (MANY ? rows <= a.small : rows > a.small)) return;
    const int r0 = rt * NB * 16;
    if (r0 >= rows) return;
    const int r1 = r0 + NB * 16 < rows ? r0 + NB * 16 : rows;
    int lo, hi;
    span_of(a, rq, r0, r1, &lo, &hi);
    const int nc = chunks_of(lo, hi, a.chunk);
    if (chunk_i >= nc) return;
    const int k0 = lo + chunk_i * a.chunk, k1 = k0 + a.chunk < hi ? k0 + a.chunk : hi;

    const int tid = threadIdx.x, lane = tid & (kWave - 1), wid = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int g = lane >> 4, c = lane & 15;
    const int back = rq.kv - rq.ql;

    // Query operands: lane (c, g) holds the D/4 values of row c that lane group g's key bytes cover.
    bf16x8 qf[NB][KS];
    int pos[NB], from[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        int r = r0 + 16 * j + c;
        r = r < rows ? r : rows - 1;
        const int t = r / a.group, head = h * a.group + (r - t * a.group);
        pos[j] = back + t;
        from[j] = a.window > 0 ? pos[j] - a.window + 1 : 0;
        const uint16_t* p = a.q + static_cast<long long>(rq.q0 + t) * a.q_stride + static_cast<long long>(head) * D + g * (D / 4);
        if (a.q_vec) {
#pragma unroll
            for (int s = 0; s < KS; ++s) qf[j][s] = *reinterpret_cast<const bf16x8*>(p + 8 * s);
        } else {
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = p[8 * s + 2 * e] | (static_cast<uint32_t>(p[8 * s + 2 * e + 1]) << 16);
                qf[j][s] = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
            }
        }
    }
    // Keys that every row sees: [all_lo, all_hi).
    const int all_hi = back + r0 / a.group + 1, all_lo = a.window > 0 ? back + (r1 - 1) / a.group - a.window + 1 : 0;

    // This wave's keys [w0, w1) and the places of its records, one a lane (at most 64: a chunk has at most 4096 keys).
    const int per = ((k1 - k0 + kWaves - 1) / kWaves + kStep - 1) / kStep * kStep;
    const int w0 = k0 + wid * per, w1 = w0 + per < k1 ? w0 + per : k1;
    const int steps = w1 > w0 ? (w1 - w0 + kStep - 1) / kStep : 0;
    long long my_off = -1;
    {
        const int key = w0 + lane * kRecTokens;
        if (key < w1) {
            const int bi = key >> a.c.page_shift;
            const int64_t row = a.rows ? a.rows[req] : req;
            const int page = row >= 0 && row < a.block_rows ? a.blocks[row * a.blocks_stride + bi] : -1;
            if (page >= 0 && page < a.c.n_pages)
                my_off = static_cast<long long>(rec_offset(a.c, page, h, (key & (a.c.page_tokens - 1)) / kRecTokens));
            else
                atomicOr(a.c.status, ELIS_DEV_BAD_PAGE);
        }
    }
    const int off_lo = static_cast<int>(my_off), off_hi = static_cast<int>(my_off >> 32);

    struct Load {
        vec k, v;
        uint32_t ks, vs;
    };
    const uint32_t lk = R::key_at(c, g * (D / 8)), lv = R::val_at(4 * g, c), lks = R::scale_k_at(c, g * (D / 4) / 32),
                   lvs = R::scale_v_at(4 * g, c * DB / 32);
    // Record x of the wave: its bytes, and whether it is there.
    auto load = [&](int x, Load& l) {
        const int lo32 = __builtin_amdgcn_readlane(off_lo, x & 63), hi32 = __builtin_amdgcn_readlane(off_hi, x & 63);
        const bool there = hi32 >= 0;
        const uint8_t* rec = a.c.pages + (there ? (static_cast<long long>(hi32) << 32 | static_cast<uint32_t>(lo32)) : 0);
        l.k = *reinterpret_cast<const vec*>(rec + lk);
        l.v = *reinterpret_cast<const vec*>(rec + lv);
        l.ks = rec[lks];
        l.vs = *reinterpret_cast<const uint32_t*>(rec + lvs);
        return there;
    };

    f32x4 o[DB][NB], lsum[NB];
    float m[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        m[j] = -INFINITY;
        lsum[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < DB; ++b) o[b][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    bf16x8 ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = static_cast<__bf16>(1.0f);
    const float sc = a.scale_log2, lag = 8.0f / sc;

    Load nx[2];
    bool nt[2] = {false, false};
    if (steps > 0) {
#pragma unroll
        for (int u = 0; u < 2; ++u) nt[u] = load(u, nx[u]);
    }
    for (int st = 0; st < steps; ++st) {
        Load cur[2] = {nx[0], nx[1]};
        const bool there[2] = {nt[0], nt[1]};
        if (st + 1 < steps) {
#pragma unroll
            for (int u = 0; u < 2; ++u) nt[u] = load(2 * st + 2 + u, nx[u]);
        }
        const int kb = w0 + st * kStep;
        f32x4 s[2][NB];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float ksc = __uint_as_float(cur[u].ks << 23);
#pragma unroll
            for (int j = 0; j < NB; ++j) s[u][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < KS; ++t) {
                const uint32_t w = cur[u].k[t];
                const u32x4 kk = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ksc, 0)),
                                  __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ksc, 1)),
                                  __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ksc, 2)),
                                  __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, ksc, 3))};
#pragma unroll
                for (int j = 0; j < NB; ++j)
                    s[u][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kk), qf[j][t], s[u][j], 0, 0, 0);
            }
        }
        // Uniform: some key of the step is not seen by some row, or holds NaN values.
        bool nan_v = false;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t x = ~cur[u].vs;  // a zero byte is a scale of 255
            nan_v = nan_v || ((x - 0x01010101u) & ~x & 0x80808080u) != 0u;
        }
        if (kb + kStep > all_hi || kb < all_lo || !there[0] || !there[1] || __ballot(nan_v) != 0ull) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t poison = 0u;  // rows whose values of this lane's columns become NaN
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = kb + 16 * u + 4 * g + i;
#pragma unroll
                    for (int j = 0; j < NB; ++j)
                        if (!there[u] || key > pos[j] || key < from[j]) s[u][j][i] = -INFINITY;
                    // values that no row may see, or that are NaN, multiply as zero
                    if (!there[u] || key >= hi || ((cur[u].vs >> (8 * i)) & 0xFFu) == 0xFFu) {
                        if constexpr (D == 128) cur[u].v[i] = 0u;
                        else cur[u].v[i >> 1] &= (i & 1) ? 0x0000FFFFu : 0xFFFF0000u;
                    }
                }
                if (there[u]) {
                    // lane (c, g) of O^T holds columns 4g..4g+3: values D/4 g ..., of scale group g D/128
                    const int grp = g * (D / 4) / 32;
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        const uint32_t w = __shfl(cur[u].vs, (x >> 2) * 16 + grp * (32 / DB), kWave);
                        const int key = kb + 16 * u + x;
                        if (((w >> (8 * (x & 3))) & 0xFFu) == 0xFFu) {
#pragma unroll
                            for (int j = 0; j < NB; ++j)
                                if (key <= pos[j] && key >= from[j]) poison |= 1u << j;
                        }
                    }
#pragma unroll
                    for (int j = 0; j < NB; ++j)
                        if (poison & (1u << j)) {
#pragma unroll
                            for (int b = 0; b < DB; ++b)
#pragma unroll
                                for (int i = 0; i < 4; ++i) o[b][j][i] = __uint_as_float(0x7FC00000u);
                        }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (((cur[u].vs >> (8 * i)) & 0xFFu) == 0xFFu) cur[u].vs &= ~(0xFFu << (8 * i));
            }
        }
        bf16x8 pf[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            float t = fmaxf(fmaxf(fmaxf(s[0][j][0], s[0][j][1]), fmaxf(s[0][j][2], s[0][j][3])),
                            fmaxf(fmaxf(s[1][j][0], s[1][j][1]), fmaxf(s[1][j][2], s[1][j][3])));
            t = quad_max(t);
            if (__ballot(t > m[j] + lag) != 0ull) {  // also the first finite maximum: m is -inf
                const float mn = fmaxf(m[j], t);
                const float w = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m[j] - mn) * sc);
                m[j] = mn;
#pragma unroll
                for (int i = 0; i < 4; ++i) lsum[j][i] *= w;
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[b][j][i] *= w;
            }
            const float ms = m[j] == -INFINITY ? 0.f : m[j] * sc;
            float p[8];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) p[4 * u + i] = __builtin_amdgcn_exp2f(fmaf(s[u][j][i], sc, -ms));
            const u32x4 pw = {pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])};
            pf[j] = __builtin_bit_cast(bf16x8, pw);
            lsum[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[j], lsum[j], 0, 0, 0);
        }
        // V^T: for every pair of a column's values, the eight keys' pairs, then even and odd value as operands of two blocks
        float vsc[8];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) vsc[4 * u + i] = scale_of(cur[u].vs, i);
#define ELIS_VPAIR(SEL)                                                                                                                \
    {                                                                                                                                  \
        uint32_t x[8];                                                                                                                 \
        _Pragma("unroll") for (int u = 0; u < 2; ++u) _Pragma("unroll") for (int i = 0; i < 4; ++i) {                                  \
            if constexpr (D == 128)                                                                                                    \
                x[4 * u + i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(cur[u].v[i], vsc[4 * u + i], SEL)); \
            else if (i & 1)                                                                                                            \
                x[4 * u + i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(cur[u].v[i >> 1], vsc[4 * u + i], 2 + ((SEL) & 1))); \
            else                                                                                                                       \
                x[4 * u + i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(cur[u].v[i >> 1], vsc[4 * u + i], (SEL) & 1)); \
        }                                                                                                                              \
        u32x4 ev, od;                                                                                                                  \
        _Pragma("unroll") for (int e = 0; e < 4; ++e) {                                                                                \
            ev[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], 0x05040100u);                                                        \
            od[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], 0x07060302u);                                                        \
        }                                                                                                                              \
        _Pragma("unroll") for (int j = 0; j < NB; ++j) {                                                                               \
            o[2 * (SEL)][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ev), pf[j], o[2 * (SEL)][j], 0, 0, 0); \
            o[2 * (SEL) + 1][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, od), pf[j], o[2 * (SEL) + 1][j], 0, 0, 0); \
        }                                                                                                                              \
    }
        ELIS_VPAIR(0)
        ELIS_VPAIR(1)
        if constexpr (D == 128) {
            ELIS_VPAIR(2)
            ELIS_VPAIR(3)
        }
#undef ELIS_VPAIR
    }

    // The four waves' parts, joined in wave order.
#pragma unroll
    for (int j = 0; j < NB; ++j)
        if (g == 0) {
            sm[wid][16 * j + c] = m[j];
            sl[wid][16 * j + c] = lsum[j][0];
        }
    __syncthreads();
    constexpr int PT = D / 16;  // values a thread joins: 16 threads a row
    const int jr = tid >> 4, jd = (tid & 15) * PT;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        if (16 * j >= r1 - r0) break;  // uniform
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sm[w][16 * j + c]);
        const float wt = m[j] == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((m[j] - top) * sc);
        if (j) __syncthreads();  // the last block has been read
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int b = 0; b < DB; b += 4) {
                const f32x4 x = {o[b][j][i] * wt, o[b + 1][j][i] * wt, o[b + 2][j][i] * wt, o[b + 3][j][i] * wt};
                *reinterpret_cast<f32x4*>(&so[wid][c][(4 * g + i) * DB + b]) = x;
            }
        __syncthreads();
        const int r = r0 + 16 * j + jr;
        if (r < r1) {
            float mt = -INFINITY, lt = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) mt = fmaxf(mt, sm[w][16 * j + jr]);
            float acc[PT];
#pragma unroll
            for (int e = 0; e < PT; ++e) acc[e] = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float mw = sm[w][16 * j + jr];
                lt += sl[w][16 * j + jr] * (mw == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((mw - mt) * sc));
#pragma unroll
                for (int e = 0; e < PT; ++e) acc[e] += so[w][jr][jd + e];
            }
            const int t = r / a.group, head = h * a.group + (r - t * a.group);
            if (nc == 1) {
                const float inv = lt == 0.f ? 1.0f : 1.0f / lt;
                uint16_t* p = a.out + static_cast<long long>(rq.q0 + t) * a.out_stride + static_cast<long long>(head) * D + jd;
                uint32_t w[PT / 2];
#pragma unroll
                for (int e = 0; e < PT; e += 2) w[e / 2] = pack_bf16x2(acc[e] * inv, acc[e + 1] * inv);
                if (a.out_vec) {
                    if constexpr (PT == 8) *reinterpret_cast<u32x4*>(p) = u32x4{w[0], w[1], w[2], w[3]};
                    else *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[1]};
                } else {
#pragma unroll
                    for (int e = 0; e < PT; ++e) p[e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
                }
            } else {
                const size_t at = part_row(a, MANY, req, h, rq.q0 + t, head, r) * a.nchunks + chunk_i;
                float* p = a.part_o + at * D + jd;
#pragma unroll
                for (int e = 0; e < PT; e += 4) *reinterpret_cast<f32x4*>(p + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
                if (jd == 0) a.part_ml[at] = float2{mt, lt};
            }
        }
    }
#endif
}

// Joins the chunks of split rows, in chunk order: one wave a row.
template <int D, bool MANY>
__global__ __launch_bounds__(kThreads) void kv_combine_kernel(KvAttnArgs a, int rows_per, int tile) {
    const int lane = threadIdx.x & (kWave - 1);
    const long long w = static_cast<long long>(blockIdx.x) * kWaves + threadIdx.x / kWave;
    int req, h, r;
    if constexpr (MANY) {
        const long long tok = w / a.n_heads;
        if (tok >= a.total_q) return;
        const int head = static_cast<int>(w - tok * a.n_heads);
        req = find_segment(a.cu, a.n, static_cast<int>(tok));
        h = head / a.group;
        r = static_cast<int>(tok - a.cu[req]) * a.group + (head - h * a.group);
    } else {
        r = static_cast<int>(w % rows_per);
        const long long u = w / rows_per;
        h = static_cast<int>(u % a.c.n_kv_heads);
        if (u / a.c.n_kv_heads >= a.n) return;
        req = static_cast<int>(u / a.c.n_kv_heads);
    }
    const Request rq = request_of(a, req);
    const int rows = rq.ql * a.group;
    if (!rq.ok || r < 0 || r >= rows || (MANY ? rows <= a.small : rows > a.small)) return;
    const int r0 = r / tile * tile, r1 = r0 + tile < rows ? r0 + tile : rows;
    int lo, hi;
    span_of(a, rq, r0, r1, &lo, &hi);
    const int nc = chunks_of(lo, hi, a.chunk);
    if (nc == 1) return;
    const int t = r / a.group, head = h * a.group + (r - t * a.group);
    const size_t at = part_row(a, MANY, req, h, rq.q0 + t, head, r) * a.nchunks;
    constexpr int PL = D / kWave;  // values a lane
    const float sc = a.scale_log2;
    float top = -INFINITY, total = 0.f, acc[PL];
#pragma unroll
    for (int e = 0; e < PL; ++e) acc[e] = 0.f;
    for (int base = 0; base < nc; base += kWave) {
        const float2 ml = base + lane < nc ? a.part_ml[at + base + lane] : float2{-INFINITY, 0.f};
        const float mt = fmaxf(top, wave_max(ml.x));
        const float old = top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((top - mt) * sc);
        const float wt = ml.x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((ml.x - mt) * sc);
        total = total * old + wave_sum(ml.y * wt);
        top = mt;
#pragma unroll
        for (int e = 0; e < PL; ++e) acc[e] *= old;
        const int n = nc - base < kWave ? nc - base : kWave;
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
            const float wi = __shfl(wt, i, kWave);
            const float* p = a.part_o + (at + base + i) * D + lane * PL;
#pragma unroll
            for (int e = 0; e < PL; ++e) acc[e] = fmaf(p[e], wi, acc[e]);
        }
    }
    const float inv = total == 0.f ? 1.0f : 1.0f / total;
    uint16_t* p = a.out + static_cast<long long>(rq.q0 + t) * a.out_stride + static_cast<long long>(head) * D + lane * PL;
#pragma unroll
    for (int e = 0; e < PL; ++e) p[e] = f32_to_bf16(acc[e] * inv);
}

template <int D>
hipError_t run(const KvAttnArgs& args, const KvAttnPlan& p, hipStream_t st) {
    KvAttnArgs a = args;
    if (p.small_rows > 0) {
        a.nchunks = p.small_chunks;
        a.chunk = p.small_chunk;
        const dim3 grid(static_cast<unsigned>(p.small_chunks), static_cast<unsigned>(a.c.n_kv_heads), static_cast<unsigned>(a.n));
        const auto f = p.small_nb == 1 ? kv_attention_kernel<D, 1, false> : p.small_nb == 2 ? kv_attention_kernel<D, 2, false> : kv_attention_kernel<D, 4, false>;
        ELIS_TRY(launch_kernel(f, grid, dim3(kThreads), 0, st, a));
        if (p.small_chunks > 1) {
            const long long waves = static_cast<long long>(a.n) * a.c.n_kv_heads * p.small_rows;
            ELIS_TRY(launch_kernel(kv_combine_kernel<D, false>, dim3(static_cast<unsigned>((waves + kWaves - 1) / kWaves)), dim3(kThreads), 0, st, a,
                                   p.small_rows, 16 * p.small_nb));
        }
    }
    if (p.many) {
        const long long tiles = (static_cast<long long>(a.max_q) * a.group + 63) / 64;
        a.chunk = p.many_chunk;
        a.nchunks = p.many_chunks;
        const dim3 grid(static_cast<unsigned>(tiles * a.nchunks), static_cast<unsigned>(a.c.n_kv_heads), static_cast<unsigned>(a.n));
        ELIS_TRY(launch_kernel(kv_attention_kernel<D, 4, true>, grid, dim3(kThreads), 0, st, a));
        if (a.nchunks > 1) {
            const long long waves = static_cast<long long>(a.total_q) * a.n_heads;
            ELIS_TRY(launch_kernel(kv_combine_kernel<D, true>, dim3(static_cast<unsigned>((waves + kWaves - 1) / kWaves)), dim3(kThreads), 0, st, a, 0, 64));
        }
    }
    return hipSuccess;
}

}  // namespace

KvAttnPlan plan_kv_attention(int n, int total_q, int max_q, int max_kv, int n_heads, int n_kv_heads) {
    KvAttnPlan p{};
    const int group = n_heads / n_kv_heads;
    const long long most = static_cast<long long>(max_q) * group;
    // one tile of 16, 32 or 64 rows holds a request, or (of longer ones) at least a single token
    const long long fit = most <= 64 ? most : group;
    if (fit <= 64) {
        p.small_nb = fit <= 16 ? 1 : fit <= 32 ? 2 : 4;
        p.small = 16 * p.small_nb;
        p.small_rows = static_cast<int>(most < p.small ? most : p.small);
        p.many = most > p.small;
        if (p.many && static_cast<long long>(n) * max_q == total_q) p.small_rows = 0;  // every request is long
        const long long per = static_cast<long long>(n) * n_kv_heads;
        long long want = (2048 + per - 1) / per;  // chunks so that about 2048 work-groups run
        long long chunk = (max_kv + want - 1) / want;
        chunk = (chunk + 127) / 128 * 128;
        chunk = chunk < 256 ? 256 : chunk > 4096 ? 4096 : chunk;
        p.small_chunk = static_cast<int>(chunk);
        p.small_chunks = static_cast<int>((max_kv + chunk - 1) / chunk);
        if (p.small_chunks < 1) p.small_chunks = 1;
    } else {
        p.many = true;
    }
    p.many_chunk = 4096;
    p.many_chunks = p.many && max_kv > 4096 ? (max_kv + 4095) / 4096 : 1;
    p.small_parts = p.small_rows > 0 && p.small_chunks > 1 ? static_cast<size_t>(n) * n_kv_heads * p.small_rows * p.small_chunks : 0;
    p.many_parts = p.many && p.many_chunks > 1 ? static_cast<size_t>(total_q) * n_heads * p.many_chunks : 0;
    return p;
}

hipError_t launch_kv_attention(KvAttnArgs a, const KvAttnPlan& p, hipStream_t st) {
    a.small = p.small;
    a.small_rows = p.small_rows;
    return a.c.d_head == 128 ? run<128>(a, p, st) : run<64>(a, p, st);
}

}  // namespace elis
