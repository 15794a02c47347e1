// Attention of new tokens over the 4-bit paged cache.
//
// Rows. The queries of one request that read the same kv head (its new tokens times the n_heads / n_kv_heads query
// heads of the group) are the rows of one product: row r is token r / G, head r % G of the group. A work-group takes 16
// NB rows of a (request, kv head) and one chunk of the keys they see; its four waves split the chunk's keys and each
// streams its own records straight from memory into registers, so nothing but the query rows (NB 2 and 4: their registers
// are what another wave on the SIMD needs) and the final merge passes through LDS. NB is 1 or 2 for requests of up to 16
// or 32 rows, single tokens above all, and 2 or 4 for tiles of longer ones.
//
// Products. As the encoder's attention: S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_16x16x32_bf16, the accumulators of
// the first being, rounded to bf16, the P^T operand of the second (lane group g holds keys 4g..4g+3 of each of a step's
// two records). The order of d inside the first product and of the rows of V^T is free, so each lane takes the 16
// consecutive bytes of a record that make its operands: of the keys D/4 consecutive values of one key (within one
// scale), of the values D/16 columns of four keys. E2M1 times a power of two is exact in bf16: one
// v_cvt_scalef32_pk_bf16_fp4 makes two operands' worth, for V^T followed by one byte permutation that pairs two keys.
//
// Softmax: running maximum and sum in fp32; the maximum lags: the accumulators are rescaled only when a score exceeds it
// by 2^8, which each lane can tell from its own scores, so the lanes of a row exchange theirs only then. It is kept as a
// whole number of powers of two, so that rescaling is exact, that of weights in bf16 too. The weights are
// rounded to bf16 for the second product (half a step, 2^-8 of each), and the rounded ones are summed.
//
// Masks. A key is seen when it is at or before the token's position, inside its window, and on a valid page. Records
// wholly seen by every row skip the test. The codes of keys that no row may see (past the end, on a bad page) are
// zeroed, so what lies there cannot matter; a group of values that holds NaN (scale 255) is multiplied as zero and
// makes NaN of exactly the rows that see it (where every row sees a record, its NaN goes through the products).
//
// Bounds. Single tokens: memory, 17/16 D bytes a key and kv head, once (48 requests of 16,000 tokens and 8 kv heads of 128:
// 183 us, 5.7 TB/s). Long prompts: the vector unit, which unpacks and takes exponentials beside
// the products (2,048 tokens of 32 heads over 16,000 keys: 480 us, 1.05 PFLOP/s; vector unit busy 61 % of it, matrix unit
// 42 %; they overlap little: two waves' 64 products and 232 vector instructions each take 1.7 us where either kind alone
// takes 0.9 and 1.1, and the kernel's 64 and 270 take 2.0). One request alone: latency. Its keys are split (chunks) and joined by a second launch.
#include <math.h>

#include <type_traits>

#include "kv_cache.h"

namespace elis {

namespace {

constexpr int kStep = 32;  // keys a wave takes at a time: two records
constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr float kLowest = -3.0e38f;  // a maximum over no keys: finite, so that differences of maxima are numbers
[[maybe_unused]] constexpr int kSpan = 32 * kWaves * kStep;  // keys whose pages the lanes of a work-group hold at a time

// Maxima in single instructions, v_maximum3_f32: fmaxf first quiets each operand's signalling NaN with an instruction of its
// own (56 more of them for a step of 64 rows). A NaN among the operands is the result. By builtins, because the compiler keeps
// the wait states between a matrix product and the first reader of its result only where it knows that reader.
__device__ __forceinline__ float max2(float x, float y) { return __builtin_elementwise_maximum(x, y); }
__device__ __forceinline__ float max3(float x, float y, float z) { return max2(max2(x, y), z); }

// s + both halves of w, a pair of bf16.
__device__ __forceinline__ float dot2(uint32_t w, float s) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, 0x3F803F80u), s, false);
#else
    return s;
#endif
}

// Byte S of w, two E2M1 values times a power of two, as a pair of bf16 (exact).
template <int S>
__device__ __forceinline__ uint32_t two_values(uint32_t w, float scale) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, S));
#else
    return 0u;
#endif
}

// Maximum over the lanes l, l^16, l^32, l^48, which hold one row's scores.
__device__ __forceinline__ float quad_max(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = max2(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return max2(__uint_as_float(b[0]), __uint_as_float(b[1]));
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

// Tile `want` of TILE rows among the requests with more than a.small rows, by all kThreads threads of the work-group (the
// two results are in LDS); false if there are fewer.
template <int TILE>
__device__ __forceinline__ bool find_tile(const KvAttnArgs& a, int want, int* tot, int* req, int* rt) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wid = tid / kWave;
    int before = 0;
    for (int base = 0; base < a.n; base += kThreads) {
        const int i = base + tid;
        int tiles = 0;
        if (i < a.n) {
            const int o0 = a.cu[i], o1 = a.cu[i + 1], ql = o1 - o0;
            if (o0 < 0 || o1 > a.total_q || o1 < o0) atomicOr(a.c.status, ELIS_DEV_BAD_CU);
            else if (ql > a.max_q) atomicOr(a.c.status, ELIS_DEV_LONG_SEQ);
            else if (ql * a.group > a.small) tiles = (ql * a.group + TILE - 1) / TILE;
        }
        int incl = tiles;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const int v = __shfl_up(incl, o, kWave);
            if (lane >= o) incl += v;
        }
        if (base) __syncthreads();  // tot has been read
        if (lane == kWave - 1) tot[wid] = incl;
        __syncthreads();
        int all = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wid) incl += tot[w];
            all += tot[w];
        }
        incl += before;
        before += all;
        if (want < incl && want >= incl - tiles) {
            *req = i;
            *rt = incl - 1 - want;
        }
        if (want < before) {
            __syncthreads();
            return true;
        }
    }
    return false;
}

__device__ __forceinline__ float scale_of(uint32_t dword, int byte) {
    return __uint_as_float(((dword >> (8 * byte)) & 0xFFu) << 23);
}

// LDS of a work-group.
template <int D, int NB>
struct Shared {
    static constexpr bool kQueries = NB > 1;  // many query rows in LDS: their registers are what another wave on the SIMD needs
    bf16x8 q[kQueries ? NB * (D / 32) * kWave : 1];
    float o[kWaves][16][D + 4];
    float m[kWaves][NB * 16], l[kWaves][NB * 16];
    int tot[kWaves], req, rt;
};

// One work-group's part, number `unit`. MANY: rows of every request with more than `small` rows, in tiles; else the
// others, one tile each, whose records nobody else reads: ONCE loads them past the caches.
template <int D, int NB, bool MANY, bool ONCE>
__device__ __forceinline__ void attend(const KvAttnArgs& a, unsigned unit, Shared<D, NB>& sh) {
#if defined(__HIP_DEVICE_COMPILE__)
    using R = Rec<D>;
    typedef typename RecRegs<D>::vec vec;
    constexpr int KS = D / 32;   // k-steps of the first product
    constexpr int DB = D / 16;   // 16-row blocks of O^T; values of a column
    constexpr bool QLDS = Shared<D, NB>::kQueries;
    constexpr int kPolicy = ONCE ? 2 : 0;  // non-temporal
    auto& so = sh.o;
    auto& sm = sh.m;
    auto& sl = sh.l;
    auto& sq = sh.q;

    // Heads fastest, then requests, tiles and chunks: the work-groups of one chunk number, which only long requests
    // have many of, spread over all XCDs (with chunks fastest 8 of them put every first chunk on one XCD: 48 -> 25 us).
    const int h = static_cast<int>(unit % a.c.n_kv_heads);
    unit /= a.c.n_kv_heads;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wid = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int g = lane >> 4, c = lane & 15;
    int req, rt = 0, chunk_i;
    if constexpr (MANY) {
        // Tiles are numbered through the requests that have more than `small` rows, last tile (most keys) first.
        chunk_i = static_cast<int>(unit % a.nchunks);
        if (!find_tile<NB * 16>(a, static_cast<int>(unit / a.nchunks), sh.tot, &sh.req, &sh.rt)) return;
        req = sh.req;
        rt = sh.rt;
    } else {
        req = static_cast<int>(unit % a.n);
        chunk_i = static_cast<int>(unit / a.n);
    }

    // The waves take the chunk's 32-key steps in turn; lane l knows the page of record l of its wave's steps (two each,
    // 32 steps at most). Without a window the keys do not depend on the lengths, and the pages are fetched along with them.
    const int64_t row = a.rows ? a.rows[req] : req;
    const bool row_ok = row >= 0 && row < a.block_rows;
    auto page_of = [&](int key) {
        const int bi = key >> a.c.page_shift;
        return row_ok && bi < a.blocks_stride ? a.blocks[row * a.blocks_stride + bi] : -1;
    };
    const int my_rec = ((wid + kWaves * (lane >> 1)) * 2 + (lane & 1)) * kRecTokens;  // its first key, from the chunk's
    int page = a.window > 0 ? 0 : page_of(chunk_i * a.chunk + my_rec);

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
    const int back = rq.kv - rq.ql;
    if (a.window > 0) page = page_of(k0 + my_rec);

    int off_lo, off_hi;  // of record `lane` of the wave's steps in the current span, or -1
    auto place = [&](int span) {
        long long off = -1;
        if (span + my_rec < k1) {
            if (page >= 0 && page < a.c.n_pages)
                off = static_cast<long long>(rec_offset(a.c, page, h, ((span + my_rec) & (a.c.page_tokens - 1)) / kRecTokens));
            else
                atomicOr(a.c.status, ELIS_DEV_BAD_PAGE);
        }
        off_lo = static_cast<int>(off);
        off_hi = static_cast<int>(off >> 32);
    };
    place(k0);

    const uint32_t lk = R::key_at(c, g * (D / 8)), lv = R::val_at(4 * g, c), lks = R::scale_k_at(c, g * (D / 4) / 32),
                   lvs = R::scale_v_at(4 * g, c * DB / 32);
    // Record x of the wave as a buffer of its bytes; one that is not there is empty and reads as zeros, so loads need no
    // condition (under one the compiler cannot tell how many are in flight, and waits for all before each step).
    auto record = [&](int x) {
        const int lo32 = __builtin_amdgcn_readlane(off_lo, x & 63);
        const int hi32 = __builtin_amdgcn_readlane(off_hi, x & 63) | ((63 - x) >> 31);  // -1 past the lanes' records
        uint8_t* rec = a.c.pages + (static_cast<long long>(hi32 & 0x7FFFFFFF) << 32 | static_cast<uint32_t>(lo32));
        return __builtin_amdgcn_make_buffer_rsrc(rec, 0, hi32 >= 0 ? R::kBytes : 0, 0x00020000);
    };
    // A step's two records in registers; the next step's are fetched while this one's are multiplied, into registers of
    // their own or (INPLACE: they are needed for 64 rows, whose step is long) into these, keys and values each as soon as
    // they have been used.
    constexpr bool INPLACE = NB == 4;
    struct Step {
        vec k[2], v[2];
        uint32_t ks[2], vs[2];
    };
    auto load_k = [&](__amdgpu_buffer_rsrc_t rec, Step& x, int u) {
        if constexpr (D == 128) x.k[u] = __builtin_amdgcn_raw_buffer_load_b128(rec, lk, 0, kPolicy);
        else x.k[u] = __builtin_amdgcn_raw_buffer_load_b64(rec, lk, 0, kPolicy);
        x.ks[u] = __builtin_amdgcn_raw_buffer_load_b32(rec, lks & ~3u, 0, kPolicy);
    };
    auto load_v = [&](__amdgpu_buffer_rsrc_t rec, Step& x, int u) {
        if constexpr (D == 128) x.v[u] = __builtin_amdgcn_raw_buffer_load_b128(rec, lv, 0, kPolicy);
        else x.v[u] = __builtin_amdgcn_raw_buffer_load_b64(rec, lv, 0, kPolicy);
        x.vs[u] = __builtin_amdgcn_raw_buffer_load_b32(rec, lvs, 0, kPolicy);
    };
    auto load = [&](int st, Step& x) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const auto rec = record(2 * st + u);
            load_k(rec, x, u);
            load_v(rec, x, u);
        }
    };
    Step x;
    load(0, x);

    // Query operands: lane (c, g) holds the D/4 values of row c that lane group g's key bytes cover.
    bf16x8 qf[QLDS ? 1 : NB][KS];
    auto token = [&](int j) {  // of row c of block j
        const int r = r0 + 16 * j + c;
        return (r < rows ? r : rows - 1) / a.group;
    };
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        int r = r0 + 16 * j + c;
        r = r < rows ? r : rows - 1;
        const int t = token(j), head = h * a.group + (r - t * a.group);
        const uint16_t* p = a.q + static_cast<long long>(rq.q0 + t) * a.q_stride + static_cast<long long>(head) * D + g * (D / 4);
        if (QLDS && j != wid) continue;  // wave j fetches block j for all
        const int jq = QLDS ? 0 : j;
        if (a.q_vec) {
#pragma unroll
            for (int s = 0; s < KS; ++s) qf[jq][s] = *reinterpret_cast<const bf16x8*>(p + 8 * s);
        } else {
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = p[8 * s + 2 * e] | (static_cast<uint32_t>(p[8 * s + 2 * e + 1]) << 16);
                qf[jq][s] = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
            }
        }
    }
    if constexpr (QLDS) {
        static_assert(NB <= kWaves, "a block of rows a wave");
        if (wid < NB) {
#pragma unroll
            for (int s = 0; s < KS; ++s) sq[(wid * KS + s) * kWave + lane] = qf[0][s];
        }
        __syncthreads();
    }
    auto query = [&](int j, int s) { return QLDS ? sq[(j * KS + s) * kWave + lane] : qf[QLDS ? 0 : j][s]; };
    // Keys that every row sees: [all_lo, all_hi).
    const int all_hi = back + r0 / a.group + 1, all_lo = a.window > 0 ? back + (r1 - 1) / a.group - a.window + 1 : 0;

    f32x4 o[DB][NB];
    float m[NB], lsum[NB];  // m in units of log2, a whole number: rescaling is exact; lsum over the lane's own keys
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        m[j] = kLowest;
        lsum[j] = 0.f;
#pragma unroll
        for (int b = 0; b < DB; ++b) o[b][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float sc = a.scale_log2;
    constexpr int UB = INPLACE ? 1 : 2;  // records whose scores are held at a time

    for (int span = k0; span < k1; span += kSpan) {  // one where rows are few: such chunks fit
        if (MANY && span > k0) {
            page = page_of(span + my_rec);
            place(span);
            load(0, x);
        }
        const int w0 = span + wid * kStep, w1 = span + kSpan < k1 ? span + kSpan : k1;
        const int steps = w0 < w1 ? (w1 - w0 + kWaves * kStep - 1) / (kWaves * kStep) : 0;
        for (int st = 0; st < steps; ++st) {
            // keeps the query rows in LDS: reads of memory that does not change would be moved out of the loop, into registers
            if constexpr (QLDS) asm volatile("" ::: "memory");
            Step next;
            if constexpr (!INPLACE) load(st + 1, next);
            const int kb = w0 + st * (kWaves * kStep);
            bool there[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) there[u] = __builtin_amdgcn_readlane(off_hi, (2 * st + u) & 63) >= 0;
            // Uniform: some key of the step is not seen by some row.
            const bool edge = kb + kStep > all_hi || kb < all_lo || !there[0] || !there[1];
            uint32_t pw[NB][4];  // the weights, as the second product's operand
            // Of two waves on a SIMD the one that multiplies goes first: the other's exponentials fill in behind (498 -> 466 us
            // for 2,048 tokens over 16,000).
            if constexpr (INPLACE) __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int u0 = 0; u0 < 2; u0 += UB) {
                f32x4 s[UB][NB];
#pragma unroll
                for (int u = 0; u < UB; ++u)
#pragma unroll
                    for (int j = 0; j < NB; ++j) s[u][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < KS; ++t) {
                    bf16x8 q[NB];
#pragma unroll
                    for (int j = 0; j < NB; ++j) q[j] = query(j, t);
#pragma unroll
                    for (int u = 0; u < UB; ++u) {
                        const uint32_t w = x.k[u0 + u][t];
                        const float ksc = scale_of(x.ks[u0 + u], lks & 3);
                        const u32x4 kk = {two_values<0>(w, ksc), two_values<1>(w, ksc), two_values<2>(w, ksc), two_values<3>(w, ksc)};
#pragma unroll
                        for (int j = 0; j < NB; ++j)
                            s[u][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kk), q[j], s[u][j], 0, 0, 0);
                    }
                }
                if constexpr (INPLACE) __builtin_amdgcn_s_setprio(0);
                if (edge) {
                    int from[NB];        // row c of block j sees the keys from, from + 1, ..., from + more; none: from lies past all
                    uint32_t more[NB];
#pragma unroll
                    for (int j = 0; j < NB; ++j) {
                        const int pos = back + token(j), f = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
                        from[j] = pos < 0 ? INT32_MAX : f;
                        more[j] = pos < 0 ? 0u : static_cast<uint32_t>(pos - f);
                    }
#pragma unroll
                    for (int u = 0; u < UB; ++u) {
                        const int v = u0 + u, kv = there[v] ? kb + 16 * v : INT32_MIN;  // a record that is not there: before all keys
                        uint32_t nan = 0u;  // of this lane's four keys, those whose values are NaN
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int key = kv + 4 * g + i;
#pragma unroll
                            for (int j = 0; j < NB; ++j)
                                if (static_cast<uint32_t>(key) - static_cast<uint32_t>(from[j]) > more[j]) s[u][j][i] = -INFINITY;
                            // values that no row may see, or that are NaN, multiply as zero
                            const bool is_nan = ((x.vs[v] >> (8 * i)) & 0xFFu) == 0xFFu;
                            if (is_nan) {
                                x.vs[v] ^= 0xFFu << (8 * i);
                                nan |= key < hi ? 1u << i : 0u;
                            }
                            if (is_nan || key >= hi) {
                                if constexpr (D == 128) x.v[v][i] = 0u;
                                else x.v[v][i >> 1] &= (i & 1) ? 0x0000FFFFu : 0xFFFF0000u;
                            }
                        }
                        if (__ballot(nan != 0u) != 0ull) {
                            // lane (c, g) of O^T holds columns 4g..4g+3: values D/4 g ..., of the scale group that lane
                            // (from_c, g') read for the keys 4g'..4g'+3
                            const int from_c = g * (D / 4) / 32 * (32 / DB);
#pragma unroll 1
                            for (int y = 0; y < 16; ++y) {
                                const uint32_t w = __shfl(nan, (y >> 2) * 16 + from_c, kWave);
#pragma unroll
                                for (int j = 0; j < NB; ++j)
                                    if (((w >> (y & 3)) & 1u) && static_cast<uint32_t>(kv + y) - static_cast<uint32_t>(from[j]) <= more[j]) {
#pragma unroll
                                        for (int b = 0; b < DB; ++b) o[b][j] = f32x4{NAN, NAN, NAN, NAN};
                                    }
                            }
                        }
                    }
                }
                if constexpr (INPLACE) load_k(record(2 * st + 2 + u0), x, u0);
                // The lanes of a row agree on m; whether to raise it each can tell from its own scores.
                float t[NB], over = -INFINITY;
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    t[j] = max2(max3(s[0][j][0], s[0][j][1], s[0][j][2]), s[0][j][3]);
                    if constexpr (UB == 2) t[j] = max3(t[j], max3(s[1][j][0], s[1][j][1], s[1][j][2]), s[1][j][3]);
                }
#pragma unroll
                for (int j = 0; j < NB; j += 2) {
                    const float x0 = fmaf(t[j], sc, -m[j]);
                    if (j + 1 < NB) over = max3(over, x0, fmaf(t[(j + 1) % NB], sc, -m[(j + 1) % NB]));
                    else over = x0;
                }
                if (__ballot(!(over <= 8.f)) != 0ull) {  // a NaN too: it is one row's alone, and may hide another row's score
#pragma unroll
                    for (int j = 0; j < NB; ++j) {
                        const float mn = max2(m[j], ceilf(quad_max(t[j]) * sc));
                        const float w = __builtin_amdgcn_exp2f(m[j] - mn);
                        m[j] = mn;
                        lsum[j] *= w;
#pragma unroll
                        for (int b = 0; b < DB; ++b)
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[b][j][i] *= w;
                        if (u0 > 0) {  // the first record's weights wait for the second product
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                pw[j][e] = pack_bf16x2(__uint_as_float(pw[j][e] << 16) * w, __uint_as_float(pw[j][e] & 0xFFFF0000u) * w);
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < NB; ++j)
#pragma unroll
                    for (int u = 0; u < UB; ++u) {
                        float p[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[u][j][i], sc, -m[j]));
                        const uint32_t w0 = pack_bf16x2(p[0], p[1]), w1 = pack_bf16x2(p[2], p[3]);
                        pw[j][2 * (u0 + u)] = w0;
                        pw[j][2 * (u0 + u) + 1] = w1;
                        lsum[j] = dot2(w1, dot2(w0, lsum[j]));
                    }
            }
            bf16x8 pf[NB];
#pragma unroll
            for (int j = 0; j < NB; ++j) pf[j] = __builtin_bit_cast(bf16x8, u32x4{pw[j][0], pw[j][1], pw[j][2], pw[j][3]});
            if constexpr (INPLACE) __builtin_amdgcn_s_setprio(1);
            // V^T: for every pair of a column's values, the eight keys' pairs, then even and odd value as operands of two blocks
            float vsc[8];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) vsc[4 * u + i] = scale_of(x.vs[u], i);
            auto pair = [&](auto sel) {
                constexpr int S = decltype(sel)::value;
                uint32_t y[8];
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float s = vsc[4 * u + i];
                        if constexpr (D == 128) y[4 * u + i] = two_values<S>(x.v[u][i], s);
                        else y[4 * u + i] = i & 1 ? two_values<2 + (S & 1)>(x.v[u][i >> 1], s) : two_values<S & 1>(x.v[u][i >> 1], s);
                    }
                u32x4 ev, od;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    ev[e] = __builtin_amdgcn_perm(y[2 * e + 1], y[2 * e], 0x05040100u);
                    od[e] = __builtin_amdgcn_perm(y[2 * e + 1], y[2 * e], 0x07060302u);
                }
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    o[2 * S][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ev), pf[j], o[2 * S][j], 0, 0, 0);
                    o[2 * S + 1][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, od), pf[j], o[2 * S + 1][j], 0, 0, 0);
                }
            };
            pair(std::integral_constant<int, 0>{});
            pair(std::integral_constant<int, 1>{});
            if constexpr (D == 128) {
                pair(std::integral_constant<int, 2>{});
                pair(std::integral_constant<int, 3>{});
            }
            if constexpr (INPLACE) {
#pragma unroll
                for (int u = 0; u < 2; ++u) load_v(record(2 * st + 2 + u), x, u);
            } else {
                x = next;
            }
        }
    }

    // The four waves' parts, joined in wave order.
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        lsum[j] += __shfl_xor(lsum[j], 16, kWave);
        lsum[j] += __shfl_xor(lsum[j], 32, kWave);
        if (g == 0) {
            sm[wid][16 * j + c] = m[j];
            sl[wid][16 * j + c] = lsum[j];
        }
    }
    __syncthreads();
    constexpr int PT = D / 16;  // values a thread joins: 16 threads a row
    const int jr = tid >> 4, jd = (tid & 15) * PT;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        if (16 * j >= r1 - r0) break;  // uniform
        float top = kLowest;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sm[w][16 * j + c]);
        const float wt = __builtin_amdgcn_exp2f(m[j] - top);
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
            float mt = kLowest, lt = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) mt = fmaxf(mt, sm[w][16 * j + jr]);
            float acc[PT];
#pragma unroll
            for (int e = 0; e < PT; ++e) acc[e] = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                lt += sl[w][16 * j + jr] * __builtin_amdgcn_exp2f(sm[w][16 * j + jr] - mt);
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
                const size_t at = kv_part_row(MANY, req, h, rq.q0 + t, head, r, a.n_heads, a.c.n_kv_heads, a.small_rows) * a.nchunks + chunk_i;
                float* p = a.part_o + at * D + jd;
#pragma unroll
                for (int e = 0; e < PT; e += 4) *reinterpret_cast<f32x4*>(p + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
                if (jd == 0) a.part_ml[at] = float2{mt, lt};
            }
        }
    }
#endif
}

constexpr int waves_per_simd(int nb) { return nb == 1 ? 4 : nb == 2 ? 3 : 2; }

template <int D, int NB, bool MANY, bool ONCE>
__global__ __launch_bounds__(kThreads, waves_per_simd(NB)) void kv_attention_kernel(KvAttnArgs a) {
    __shared__ __attribute__((aligned(16))) Shared<D, NB> sh;
    attend<D, NB, MANY, ONCE>(a, blockIdx.x, sh);
}

// Both at once: neither waits for the other's last work-groups. The long requests' tiles come first, the single tokens fill
// in behind (two prompts of up to 512 tokens beside 30 tokens: 37 us, the tokens among the tiles 43, before them 42).
template <int D, int NB, int NBM, bool ONCE>
__global__ __launch_bounds__(kThreads, waves_per_simd(NBM)) void kv_attention_mixed_kernel(KvAttnArgs a, KvAttnMany m) {
    union Both {
        Shared<D, NBM> many;
        Shared<D, NB> small;
    };
    __shared__ __attribute__((aligned(16))) char raw[sizeof(Both)];
    Both& sh = *reinterpret_cast<Both*>(raw);
    if (blockIdx.x < static_cast<unsigned>(m.units)) {
        attend<D, NBM, true, false>(m.of(a, D), blockIdx.x, sh.many);
    } else {
        attend<D, NB, false, ONCE>(a, blockIdx.x - m.units, sh.small);
    }
}

// Joins the chunks of split rows, in an order that depends on their number alone. WAVES waves a row, each taking every
// WAVES-th chunk: with one wave a row of 118 chunks took 38 us, its loads one behind the other.
// A wave past the last row reads nothing: its place in the chunk results may lie behind them.
template <int D, int WAVES>
__global__ __launch_bounds__(kThreads) void kv_combine_kernel(KvAttnArgs a, KvAttnMany m, KvJoins joins, int small_tile) {
    __shared__ __attribute__((aligned(16))) float part[WAVES > 1 ? kWaves : 1][D];
    const int lane = threadIdx.x & (kWave - 1), wid = threadIdx.x / kWave;
    const KvJoinRow x = kv_join_row(static_cast<long long>(blockIdx.x) * (kWaves / WAVES) + wid / WAVES, joins, a.small_rows, a.n_heads, a.c.n_kv_heads);
    if (!x.any) return;
    const int wi = wid % WAVES;
    const bool many = x.many;
    const int tile = many ? m.tile : small_tile;
    int req = x.req, h = x.h, r = x.r;
    if (many) a = m.of(a, D);
    // Where the results are does not depend on the lengths: the first are requested along with them (one request of 30,001
    // tokens 13.8 -> 13.0 us).
    const size_t at = kv_part_row(many, req, h, x.tok, x.head, r, a.n_heads, a.c.n_kv_heads, a.small_rows) * a.nchunks;
    constexpr int PL = D / kWave;  // values a lane
    constexpr int AHEAD = 8;       // chunks a wave fetches at a time, the first before their weights are known
    typedef float fvec __attribute__((ext_vector_type(PL)));
    fvec v[AHEAD];
    auto fetch = [&](int i0, int last) {
#pragma unroll
        for (int y = 0; y < AHEAD; ++y) {
            const int i = i0 + y * WAVES;
            v[y] = *reinterpret_cast<const fvec*>(a.part_o + (at + (i < last ? i : last)) * D + lane * PL);
        }
    };
    float2 ml{};
    auto begin = [&] {
        ml = a.part_ml[at + (lane < a.nchunks ? lane : 0)];
        fetch(wi, a.nchunks - 1);
    };
    const bool early = many || r < a.group;  // rows that a single token has
    if (early) begin();
    if (many) {
        req = find_segment(a.cu, a.n, x.tok);
        h = x.head / a.group;
        r = (x.tok - a.cu[req]) * a.group + (x.head - h * a.group);
    }
    const Request rq = request_of(a, req);
    const int rows = rq.ql * a.group;
    if (!rq.ok || r < 0 || r >= rows || (many ? rows <= a.small : rows > a.small)) return;
    const int r0 = r / tile * tile, r1 = r0 + tile < rows ? r0 + tile : rows;
    int lo, hi;
    span_of(a, rq, r0, r1, &lo, &hi);
    const int nc = chunks_of(lo, hi, a.chunk);
    if (nc == 1) return;  // every return is the same for the waves of a row
    if (!early) begin();
    float top = kLowest, total = 0.f;
    fvec acc = 0.f;
    for (int base = 0; base < nc; base += kWave) {
        const int n = nc - base < kWave ? nc - base : kWave;
        if (base) {
            ml = a.part_ml[at + base + (lane < n ? lane : 0)];
            fetch(base + wi, base + n - 1);
        }
        if (lane >= n) ml = float2{kLowest, 0.f};
        const float mt = fmaxf(top, wave_max(ml.x));
        const float old = __builtin_amdgcn_exp2f(top - mt), wt = __builtin_amdgcn_exp2f(ml.x - mt);
        total = total * old + wave_sum(ml.y * wt);
        acc *= old;
        top = mt;
        for (int i0 = wi; i0 < n; i0 += AHEAD * WAVES) {
            if (i0 > wi) fetch(base + i0, base + n - 1);
#pragma unroll
            for (int y = 0; y < AHEAD; ++y) {
                const int i = i0 + y * WAVES;
                if (i < n) acc += v[y] * __shfl(wt, i, kWave);  // uniform
            }
        }
    }
    if constexpr (WAVES > 1) {
#pragma unroll
        for (int e = 0; e < PL; ++e) part[wid][lane * PL + e] = acc[e];
        __syncthreads();
        if (wi != 0) return;
#pragma unroll
        for (int x = 1; x < WAVES; ++x)
#pragma unroll
            for (int e = 0; e < PL; ++e) acc[e] += part[wid + x][lane * PL + e];
    }
    const float inv = total == 0.f ? 1.0f : 1.0f / total;
    const int t = r / a.group;
    uint16_t* p = a.out + static_cast<long long>(rq.q0 + t) * a.out_stride + static_cast<long long>(h * a.group + (r - t * a.group)) * D + lane * PL;
#pragma unroll
    for (int e = 0; e < PL; ++e) p[e] = f32_to_bf16(acc[e] * inv);
}

template <int D>
constexpr int kNbMost = D == 128 ? 4 : 2;

template <int D>
hipError_t run(const KvAttnArgs& args, const KvAttnPlan& p, hipStream_t st) {
    KvAttnArgs a = args;  // as the short requests' launch takes it
    a.nchunks = p.small_chunks;
    a.chunk = p.small_chunk;
    const unsigned heads = static_cast<unsigned>(a.c.n_kv_heads);
    const unsigned small = p.small_rows > 0 ? heads * a.n * p.small_chunks : 0, many = heads * p.many_tiles * p.many_chunks;
    const KvAttnMany m{static_cast<int>(many), p.many_chunk, p.many_chunks, 16 * p.many_nb, p.small_parts};  // both may have chunk results at once
    if (small) {
        const auto go = [&](auto nb, auto once) {
            constexpr int NB = decltype(nb)::value;
            constexpr bool ONCE = decltype(once)::value;
            if (!many) return launch_kernel(kv_attention_kernel<D, NB, false, ONCE>, dim3(small), dim3(kThreads), 0, st, a);
            const auto f = p.many_nb == 4 ? kv_attention_mixed_kernel<D, NB, kNbMost<D>, ONCE> : kv_attention_mixed_kernel<D, NB, 2, ONCE>;
            return launch_kernel(f, dim3(small + many), dim3(kThreads), 0, st, a, m);
        };
        const std::integral_constant<int, 1> one{};
        const std::integral_constant<int, 2> two{};
        ELIS_TRY(p.once ? (p.small_nb == 1 ? go(one, std::true_type{}) : go(two, std::true_type{}))
                        : (p.small_nb == 1 ? go(one, std::false_type{}) : go(two, std::false_type{})));
    } else if (many) {
        const auto f = p.many_nb == 4 ? kv_attention_kernel<D, kNbMost<D>, true, false> : kv_attention_kernel<D, 2, true, false>;
        ELIS_TRY(launch_kernel(f, dim3(many), dim3(kThreads), 0, st, m.of(a, D)));
    }
    const KvJoins joins = kv_joins(p, a.n, a.total_q, a.n_heads, a.c.n_kv_heads);
    if (joins.all == 0) return hipSuccess;
    const auto f = joins.wide ? kv_combine_kernel<D, kWaves> : kv_combine_kernel<D, 1>;
    const unsigned grid = static_cast<unsigned>(joins.wide ? joins.all : (joins.all + kWaves - 1) / kWaves);
    return launch_kernel(f, dim3(grid), dim3(kThreads), 0, st, a, m, joins, 16 * p.small_nb);
}

}  // namespace

hipError_t launch_kv_attention(KvAttnArgs a, const KvAttnPlan& p, hipStream_t st) {
    a.small = p.small;
    a.small_rows = p.small_rows;
    return a.c.d_head == 128 ? run<128>(a, p, st) : run<64>(a, p, st);
}

}  // namespace elis
