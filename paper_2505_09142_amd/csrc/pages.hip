// Page pool: block tables and slot maps of a batch, built on the device out of its lengths.
//
// The pool is a stack of free page ids and, per job slot, the pages that the job holds in token order. grow gives
// every job of the call the pages that its length after the step needs: with need_i = max(0, ceil(len_i / P) - held_i)
// and off_i the exclusive prefix sum of need over the call, job i takes the stack's entries top - off_i, top - off_i - 1,
// ..., if off_i + need_i pages are there (so the jobs served are a prefix of those that need any, in the order of the
// call: the selection's priority order). The slot of the token at position p is table[p / P] * P + p % P. trim takes the
// pages past a shorter length back, in the order that makes it the exact inverse of grow.
//
// Both are a scan over the batch by one work-group and then independent work for every job: its new table entries, its
// row of the batch's block table, and a slot for each new token. Small batches do both in one launch (pages_small_kernel:
// the entries in LDS, the work spread over all threads); larger ones leave what the second part needs in the pool's
// scratch (for each entry of the call the stack place of its first page that moves, and its pages before and after) and
// hand each job's part to a work-group (or several) of a second launch. Bound by latency: a few dependent loads.
#include "kernels.h"

namespace elis {

namespace {

constexpr int kScan = 1024;   // threads of the scan
constexpr int kEach = 2;      // entries a thread of it holds at a time (grow and trim of 200 entries: 1 / 2 / 4 of them 11.0 / 11.7 /
                              // 13.3 us, of 2,048: 21.1 / 20.0 / 22.1, of 20,000: 152 / 138 / 150)
constexpr int kSmall = 128;   // entries up to which one launch does all,
// with at most so many cells and slots to write. Grow and trim with the grow in one launch and in two, GPU's time / among other
// calls: 12,900 of 64 jobs a step 9.7 / 10.0 and 9.2 / 13.0 us, 19,000 of 20 new jobs 20.2 / 20.1 and 11.1 / 13.1.
constexpr int kSmallWork = 16384;
constexpr int kFill = 256;    // threads of a work-group of the second launch
constexpr int kFillGroups = 65536;  // of them in a row of the grid: a row has fewer than 2^32 threads, a call up to 2^29 entries
constexpr int32_t kClaim = INT32_MIN;  // held[s] with its top bit set: named by an entry of the running call

struct FillArgs {
    PagePoolView p;
    const int32_t* slots;
    const int32_t* lens;
    const int32_t* cu;   // grow: new tokens of each entry
    int n, total, width;
    int32_t* blocks;     // or null
    int32_t* map;        // or null
};

__device__ __forceinline__ int clamp_held(int32_t h, int max_pages) {
    h &= ~kClaim;
    return h < 0 ? 0 : h > max_pages ? max_pages : h;
}
__device__ __forceinline__ int clamp_count(int32_t c, int n_pages) { return c < 0 ? 0 : c > n_pages ? n_pages : c; }

// Entry i's part, shared by `step` threads of which this is number `t`. first: stack place of its first page that
// moves; h0, h1: its pages before and after.
template <bool GROW>
__device__ __forceinline__ void pages_fill(const FillArgs& a, int i, int32_t s, int first, int h0, int h1, int t, int step) {
    if (s < 0 || s >= a.p.max_jobs) {
        if (GROW && a.blocks)
            for (int j = t; j < a.width; j += step) a.blocks[static_cast<size_t>(i) * a.width + j] = -1;
        h0 = h1 = 0;
        s = 0;
    }
    int32_t* row = a.p.table + static_cast<size_t>(s) * a.p.max_pages;
    if constexpr (GROW) {
        auto page = [&](int j) { return j < h0 ? row[j] : a.p.free_pages[first - (j - h0)]; };  // j < h1
        for (int j = h0 + t; j < h1; j += step) row[j] = a.p.free_pages[first - (j - h0)];
        if (a.blocks && h1 > 0) {
            int32_t* out = a.blocks + static_cast<size_t>(i) * a.width;
            for (int j = t; j < a.width; j += step) out[j] = j < h1 ? page(j) : -1;
        } else if (a.blocks) {
            for (int j = t; j < a.width; j += step) a.blocks[static_cast<size_t>(i) * a.width + j] = -1;
        }
        if (a.map) {
            const int o0 = a.cu[i], o1 = a.cu[i + 1];
            if (o0 < 0 || o1 > a.total || o1 < o0) return;  // flagged by the scan
            const long long before = static_cast<long long>(a.lens[i]) - (o1 - o0);
            for (int q = t; q < o1 - o0; q += step) {
                const long long pos = before + q;
                int32_t at = -1;
                if (pos >= 0) {
                    const int j = static_cast<int>(pos >> a.p.page_shift);
                    if (j < h1) at = (page(j) << a.p.page_shift) + static_cast<int>(pos & (a.p.page_tokens - 1));
                }
                a.map[o0 + q] = at;
            }
        }
    } else {
        for (int j = h1 + t; j < h0; j += step) {
            const int to = first - (j - h1);
            if (to >= 0 && to < a.p.n_pages) a.p.free_pages[to] = row[j];
        }
    }
}

// Pages that entry (len, new tokens [o0, o1)) of a job that holds h0 moves, and the content errors it shows.
template <bool GROW>
__device__ __forceinline__ int pages_move(const FillArgs& a, int i, int len, int o0, int o1, int h0, uint32_t* bad) {
    if (GROW && a.map &&
        (o0 < 0 || o1 < o0 || o1 > a.total || (i == 0 && o0 != 0) || (i == a.n - 1 && o1 != a.total) || o1 - o0 > len))
        *bad |= ELIS_DEV_BAD_CU;
    const long long want = (static_cast<long long>(len) + a.p.page_tokens - 1) >> a.p.page_shift;
    if (len < 0) {
        *bad |= ELIS_DEV_BAD_SLOT;
        return 0;
    }
    if (GROW && want > a.p.max_pages) {
        *bad |= ELIS_DEV_LONG_SEQ;
        return 0;
    }
    return GROW ? (want > h0 ? static_cast<int>(want) - h0 : 0) : (want < h0 ? h0 - static_cast<int>(want) : 0);
}

// Inclusive sum over the threads of a work-group of kScan, and the total.
__device__ __forceinline__ int block_scan(int v, int32_t* wave_tot, int* total) {
    constexpr int kW = kScan / kWave;
    const int lane = threadIdx.x & (kWave - 1), wid = threadIdx.x / kWave;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const int u = __shfl_up(v, o, kWave);
        if (lane >= o) v += u;
    }
    if (lane == kWave - 1) wave_tot[wid] = v;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kW; ++w) {
        const int u = wave_tot[w];
        if (w < wid) before += u;
        all += u;
    }
    *total = all;
    return v + before;
}

// Up to kSmall entries, everything in one launch.
template <bool GROW>
__global__ __launch_bounds__(kScan) void pages_small_kernel(FillArgs a) {
    __shared__ int32_t wave_tot[kScan / kWave];
    __shared__ int32_t slot[kSmall], excl[kSmall], h0s[kSmall], h1s[kSmall], lens[kSmall], cu[kSmall + 1], again[kSmall];
    __shared__ int32_t taken_s, more_s;
    __shared__ uint32_t bad_s;
    const int tid = threadIdx.x, i = tid;
    if (tid == 0) {
        bad_s = 0u;
        taken_s = more_s = 0;
    }
    const int count = clamp_count(a.p.state[1], a.p.n_pages);
    uint32_t bad = 0u;
    int32_t s = -1;
    int len = 0, h0 = 0, o0 = 0, o1 = 0;
    if (i < kSmall) {
        const int ic = i < a.n ? i : a.n - 1;
        s = a.slots[ic];
        len = a.lens[ic];
        if (GROW && a.map) {
            o0 = a.cu[ic];
            o1 = a.cu[ic + 1];
            if (i < a.n) cu[i] = o0;  // the place behind them is the last entry's alone
            if (i == a.n - 1) cu[a.n] = o1;
        }
        if (i >= a.n) {
            s = -1;
        } else if (s < 0 || s >= a.p.max_jobs) {
            bad |= ELIS_DEV_BAD_SLOT;
            s = -1;
        } else {
            h0 = clamp_held(a.p.held[s], a.p.max_pages);
        }
        slot[i] = s;
        lens[i] = len;
        h0s[i] = h0;
        again[i] = 0;
    }
    __syncthreads();
    // A slot that an earlier entry names too: that one is served. Each wave compares eight entries with all (an entry's
    // thread alone, with all before it, took 1.2 us longer).
    const int wid = tid / kWave, lane = tid & (kWave - 1);
    static_assert(kSmall == 2 * kWave && kSmall == 8 * (kScan / kWave), "two entries a lane, eight a wave");
    {
        const int s0 = slot[lane], s1 = slot[lane + kWave];
        bool d0 = false, d1 = false;
        for (int j = 8 * wid; j < 8 * wid + 8 && j < a.n; ++j) {
            const int sj = slot[j];
            d0 |= sj == s0 && j < lane;
            d1 |= sj == s1 && j < lane + kWave;
        }
        if (d0) again[lane] = 1;
        if (d1) again[lane + kWave] = 1;
    }
    __syncthreads();
    int move = 0;
    if (i < a.n && s >= 0) {
        if (again[i]) bad |= ELIS_DEV_BAD_SLOT;
        else move = pages_move<GROW>(a, i, len, o0, o1, h0, &bad);
    }
    int total;
    const int incl = block_scan(move, wave_tot, &total);
    const int top = (GROW ? count : count + total) - 1;  // stack place of the first page that moves
    auto move_page = [&](int32_t of, int j, int at) {     // page j of job slot `of`
        int32_t* cell = a.p.table + static_cast<size_t>(of) * a.p.max_pages + j;
        if (GROW) *cell = a.p.free_pages[at];
        else if (at >= 0 && at < a.p.n_pages) a.p.free_pages[at] = *cell;
    };
    int h1 = h0;
    if (i < a.n) {
        if (GROW) {
            const bool fits = move == 0 || incl <= count;
            if (!fits) bad |= ELIS_DEV_NO_PAGES;
            else h1 = h0 + move;
            if (total > count && move > 0 && fits) atomicMax(&taken_s, incl);
        } else {
            h1 = h0 - move;
        }
        excl[i] = incl - move;
        h1s[i] = h1;
        if (h1 != h0) {
            a.p.held[s] = h1;
            move_page(s, GROW ? h0 : h1, top - (incl - move));  // the only one, in a step of a token each
            if (move > 1) more_s = 1;
        }
    }
    if (bad) atomicOr(&bad_s, bad);
    __syncthreads();
    if (tid == 0) {
        const int now = GROW ? count - (total > count ? taken_s : total) : count + total;
        a.p.state[1] = now < a.p.n_pages ? now : a.p.n_pages;
        if (bad_s) atomicOr(reinterpret_cast<uint32_t*>(&a.p.state[0]), bad_s);
    }
    auto page = [&](int k, int j) {  // of entry k, j < h1
        return j < h0s[k] ? a.p.table[static_cast<size_t>(slot[k]) * a.p.max_pages + j] : a.p.free_pages[top - excl[k] - (j - h0s[k])];
    };
    if (more_s) {  // the other pages that move, one a thread (a wave an entry took 4 us longer for 100 new requests)
        for (int m = tid; m < total; m += kScan) {
            const int k = find_segment(excl, a.n, m), j = (GROW ? h0s[k] : h1s[k]) + m - excl[k];
            if (j >= (GROW ? h1s[k] : h0s[k])) break;  // entries that the free pages do not reach for, to the last
            move_page(slot[k], j, top - m);
        }
    }
    if (GROW && a.blocks) {
        // Cell x is (x / width, x % width). Each load's address is chosen, not the load: eight are in flight at once. (More
        // of them, or the comparison of slots unrolled, cost more in fetching the code than they save: 7.6 -> 11.8 us.)
        constexpr int U = 8;
        const int cells = a.n * a.width, dk = kScan / a.width, dj = kScan - dk * a.width;
        int k = tid / a.width, j = tid - k * a.width;
        for (int x = tid; x < cells; x += U * kScan) {
            int32_t v[U];
            bool in[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                in[u] = x + u * kScan < cells;
                const int kc = in[u] ? k : 0, h0k = h0s[kc];
                const bool has = in[u] && j < h1s[kc];
                const int32_t* from = a.slots;
                if (has) from = j < h0k ? a.p.table + static_cast<size_t>(slot[kc]) * a.p.max_pages + j : a.p.free_pages + (top - excl[kc] - (j - h0k));
                v[u] = *from;
                v[u] = has ? v[u] : -1;
                k += dk;
                j += dj;
                if (j >= a.width) {
                    j -= a.width;
                    ++k;
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (in[u]) a.blocks[x + u * kScan] = v[u];
        }
    }
    if (GROW && a.map) {
        for (int t = tid; t < a.total; t += kScan) {
            const int k = find_segment(cu, a.n, t);
            const int c0 = cu[k], c1 = cu[k + 1];
            if (t < c0 || t >= c1) continue;  // malformed offsets, flagged above
            const long long pos = static_cast<long long>(lens[k]) - (c1 - c0) + (t - c0);
            int32_t at = -1;
            if (pos >= 0) {
                const long long j = pos >> a.p.page_shift;
                if (j < h1s[k]) at = (page(k, static_cast<int>(j)) << a.p.page_shift) + static_cast<int>(pos & (a.p.page_tokens - 1));
            }
            a.map[t] = at;
        }
    }
}

// Any number of entries: the scan alone.
template <bool GROW>
__global__ __launch_bounds__(kScan) void pages_scan_kernel(FillArgs a) {
    __shared__ int32_t wave_tot[kScan / kWave];
    __shared__ int32_t taken_s;
    __shared__ uint32_t bad_s;
    const int tid = threadIdx.x;
    if (tid == 0) {
        bad_s = 0u;
        taken_s = 0;
    }
    const int count = clamp_count(a.p.state[1], a.p.n_pages);
    uint32_t bad = 0u;
    // First pass: claim every slot (a slot named twice keeps its first claim), pages that move per entry, their prefix.
    int carry = 0, taken = 0;
    for (int base = 0; base < a.n; base += kEach * kScan) {
        const int i0 = base + kEach * tid;
        int32_t s[kEach];
        int len[kEach], o[kEach + 1] = {}, h0[kEach], move[kEach], sum = 0;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int i = i0 + e < a.n ? i0 + e : a.n - 1;  // loads without a condition are all in flight at once
            s[e] = a.slots[i];
            len[e] = a.lens[i];
        }
        if (GROW && a.map) {
#pragma unroll
            for (int e = 0; e <= kEach; ++e) o[e] = a.cu[i0 + e < a.n ? i0 + e : a.n];
        }
        int32_t old[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const bool ok = i0 + e < a.n && s[e] >= 0 && s[e] < a.p.max_jobs;
            if (!ok) s[e] = -1;
            old[e] = ok ? atomicOr(&a.p.held[s[e]], kClaim) : 0;
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            move[e] = h0[e] = 0;
            if (i0 + e < a.n) {
                if (s[e] < 0 || (old[e] & kClaim)) bad |= ELIS_DEV_BAD_SLOT;
                if (s[e] >= 0) {
                    h0[e] = clamp_held(old[e], a.p.max_pages);
                    if (!(old[e] & kClaim)) move[e] = pages_move<GROW>(a, i0 + e, len[e], o[e], o[e + 1], h0[e], &bad);
                }
            }
            sum += move[e];
        }
        int all;
        int incl = block_scan(sum, wave_tot, &all) + carry - sum;
        carry += all;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int i = i0 + e, first = count - 1 - incl;  // trim: the total is added once it is known
            incl += move[e];
            int h1 = GROW ? h0[e] : h0[e] - move[e];
            if (GROW) {
                if (move[e] == 0 || incl <= count) h1 += move[e];
                else bad |= ELIS_DEV_NO_PAGES;
                if (h1 != h0[e]) taken = incl;
            }
            if (i < a.n) {
                int4* out = reinterpret_cast<int4*>(a.p.scratch + 4 * static_cast<size_t>(i));
                const int4 v = {first, h0[e], h1, 0};
                if (a.p.scratch_vec) *out = v;
                else {
                    a.p.scratch[4 * static_cast<size_t>(i)] = v.x;
                    a.p.scratch[4 * static_cast<size_t>(i) + 1] = v.y;
                    a.p.scratch[4 * static_cast<size_t>(i) + 2] = v.z;
                }
            }
        }
        __syncthreads();  // wave_tot is free
    }
    // Where the free pages reach for all, they are the sum; a maximum over 1,024 threads costs 3.5 us.
    if (carry > count && taken) atomicMax(&taken_s, taken);
    if (bad) atomicOr(&bad_s, bad);
    __syncthreads();
    if (tid == 0) {
        const int now = GROW ? count - (carry > count ? taken_s : carry) : count + carry;
        a.p.state[1] = now < a.p.n_pages ? now : a.p.n_pages;
        if (!GROW) a.p.scratch[4 * static_cast<size_t>(a.p.max_jobs)] = carry;
        if (bad_s) atomicOr(reinterpret_cast<uint32_t*>(&a.p.state[0]), bad_s);
    }
}

template <bool GROW>
__global__ __launch_bounds__(kFill) void pages_fill_kernel(FillArgs a, int parts) {
    const int group = blockIdx.x / parts, part = blockIdx.x - group * parts, i = blockIdx.y * kFillGroups + group;
    if (i >= a.n) return;
    const int32_t* e = a.p.scratch + 4 * static_cast<size_t>(i);
    const int first = e[0] + (GROW ? 0 : a.p.scratch[4 * static_cast<size_t>(a.p.max_jobs)]), h0 = e[1], h1 = e[2];
    const int32_t s = a.slots[i];
    // The claim of the scan ends: with the new count, or, where nothing moves, by itself (an entry whose slot an earlier
    // one had claimed moves nothing).
    if (part == 0 && threadIdx.x == 0 && s >= 0 && s < a.p.max_jobs) {
        if (h1 != h0) a.p.held[s] = h1;
        else atomicAnd(&a.p.held[s], ~kClaim);
    }
    pages_fill<GROW>(a, i, s, first, h0, h1, part * kFill + threadIdx.x, parts * kFill);
}

__global__ __launch_bounds__(kFill) void pages_init_kernel(PagePoolView p) {
    const int i = blockIdx.x * kFill + threadIdx.x;
    if (i == 0) {
        p.state[0] = 0;
        p.state[1] = p.n_pages;
    }
    if (i < p.n_pages) p.free_pages[i] = p.n_pages - 1 - i;
    if (i < p.max_jobs) p.held[i] = 0;
}

template <bool GROW>
hipError_t launch_pages(const FillArgs& a, hipStream_t st) {
    const long long work = GROW ? static_cast<long long>(a.map ? a.total : 0) + (a.blocks ? static_cast<long long>(a.n) * a.width : 0) : 0;
    if (a.n <= kSmall && work <= kSmallWork) return launch_kernel(pages_small_kernel<GROW>, dim3(1), dim3(kScan), 0, st, a);
    ELIS_TRY(launch_kernel(pages_scan_kernel<GROW>, dim3(1), dim3(kScan), 0, st, a));
    // About two elements a thread (1 / 2 / 4 / 16 of them: 20 jobs of 1,500 tokens 11.1 / 11.5 / 12.1 / 12.1 us, two of 100,000
    // 15.8 / 15.9 / 15.9 / 19.2, 1,000 jobs a step 14.7 / 14.1 / 14.2 / 14.1).
    long long parts = work / (static_cast<long long>(a.n) * 2 * kFill);
    parts = parts < 1 ? 1 : parts > 64 ? 64 : parts;
    if (parts * a.n > kFillGroups) parts = 1;
    const int row = a.n < kFillGroups ? a.n : kFillGroups;
    return launch_kernel(pages_fill_kernel<GROW>, dim3(static_cast<unsigned>(parts * row), static_cast<unsigned>((a.n - 1) / kFillGroups + 1)), dim3(kFill), 0,
                         st, a, static_cast<int>(parts));
}

}  // namespace

hipError_t launch_pages_init(PagePoolView p, hipStream_t st) {
    const int n = p.n_pages > p.max_jobs ? p.n_pages : p.max_jobs;
    return launch_kernel(pages_init_kernel, dim3(static_cast<unsigned>((n + static_cast<long long>(kFill) - 1) / kFill)), dim3(kFill), 0, st, p);
}

hipError_t launch_pages_grow(PagePoolView p, const int32_t* slots, const int32_t* lens, const int32_t* cu, int n, int total, int width,
                             int32_t* blocks, int32_t* map, hipStream_t st) {
    return launch_pages<true>(FillArgs{p, slots, lens, cu, n, total, width, blocks, map}, st);
}

hipError_t launch_pages_trim(PagePoolView p, const int32_t* slots, const int32_t* lens, int n, hipStream_t st) {
    return launch_pages<false>(FillArgs{p, slots, lens, nullptr, n, 0, 0, nullptr, nullptr}, st);
}

}  // namespace elis
