// Page pool: block tables and slot maps of a batch, built on the device out of its lengths.
//
// The pool is a stack of free page ids and, per job slot, the pages that the job holds in token order. grow gives
// every job of the call the pages that its length after the step needs: with need_i = max(0, ceil(len_i / P) - held_i)
// and off_i the exclusive prefix sum of need over the call, job i takes the stack's entries top - off_i, top - off_i - 1,
// ..., if off_i + need_i pages are there (so the jobs served are a prefix of those that need any, in the order of the
// call: the selection's priority order). The slot of the token at position p is table[p / P] * P + p % P. trim takes the
// pages past a shorter length back, in the order that makes it the exact inverse of grow.
//
// Both are a scan over the batch (one work-group, pages_scan_kernel) and then independent work for every job
// (pages_fill): its new table entries, its row of the batch's block table, and a slot for each new token. Small
// batches do both in the one work-group's launch; larger ones hand each job's part to a work-group (or several) of a
// second launch. What the second part needs of the first is left in the pool's scratch: for each entry of the call
// the stack place of its first page that moves, and its pages before the call.
#include "kernels.h"

namespace elis {

namespace {

constexpr int kScan = 1024;   // threads of the scan
constexpr int kFill = 256;    // threads of a work-group of the second launch
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

template <bool GROW, bool FUSED>
__global__ __launch_bounds__(kScan) void pages_scan_kernel(FillArgs a) {
    constexpr int kW = kScan / kWave;
    __shared__ int32_t wave_tot[kW];
    __shared__ int32_t sh_first[FUSED ? kScan : 1], sh_h0[FUSED ? kScan : 1], sh_h1[FUSED ? kScan : 1], sh_slot[FUSED ? kScan : 1];
    __shared__ int32_t taken_s;
    __shared__ uint32_t bad_s;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wid = tid / kWave;
    if (tid == 0) {
        bad_s = 0u;
        taken_s = 0;
    }
    const int count = clamp_count(a.p.state[1], a.p.n_pages);
    uint32_t bad = 0u;
    __syncthreads();
    // First pass: claim every slot (a slot named twice keeps its first claim), pages that move per entry, their prefix.
    int carry = 0, taken = 0;
    for (int base = 0; base < a.n; base += kScan) {
        const int i = base + tid;
        int32_t s = -1;
        int move = 0, h0 = 0;
        if (i < a.n) {
            s = a.slots[i];
            const int len = a.lens[i];
            if (s < 0 || s >= a.p.max_jobs) {
                bad |= ELIS_DEV_BAD_SLOT;
                s = -1;
            } else {
                const int32_t old = atomicOr(&a.p.held[s], kClaim);
                h0 = clamp_held(old, a.p.max_pages);
                const long long want = (static_cast<long long>(len) + a.p.page_tokens - 1) >> a.p.page_shift;
                if (old & kClaim) {
                    bad |= ELIS_DEV_BAD_SLOT;
                } else if (len < 0) {
                    bad |= ELIS_DEV_BAD_SLOT;
                } else if (GROW && want > a.p.max_pages) {
                    bad |= ELIS_DEV_LONG_SEQ;
                } else {
                    move = GROW ? (want > h0 ? static_cast<int>(want) - h0 : 0) : (want < h0 ? h0 - static_cast<int>(want) : 0);
                }
            }
            if (GROW && a.map) {
                const int o0 = a.cu[i], o1 = a.cu[i + 1];
                if (o0 < 0 || o1 < o0 || o1 > a.total || (i == 0 && o0 != 0) || (i == a.n - 1 && o1 != a.total) || o1 - o0 > len)
                    bad |= ELIS_DEV_BAD_CU;
            }
        }
        int incl = move;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const int v = __shfl_up(incl, o, kWave);
            if (lane >= o) incl += v;
        }
        if (lane == kWave - 1) wave_tot[wid] = incl;
        __syncthreads();
        int before = carry, all = 0;
#pragma unroll
        for (int w = 0; w < kW; ++w) {
            const int v = wave_tot[w];
            if (w < wid) before += v;
            all += v;
        }
        incl += before;
        carry += all;
        const int off = incl - move;
        int first, h1;
        if constexpr (GROW) {
            const bool fits = move == 0 || incl <= count;
            if (!fits) bad |= ELIS_DEV_NO_PAGES;
            h1 = fits ? h0 + move : h0;
            first = count - 1 - off;
            if (move > 0 && fits && incl > taken) taken = incl;
        } else {
            h1 = h0 - move;
            first = count - 1 - off;  // the total is added once it is known
        }
        if (i < a.n) {
            if constexpr (FUSED) {
                sh_first[i] = first;
                sh_h0[i] = h0;
                sh_h1[i] = h1;
                sh_slot[i] = s;
            } else {
                a.p.scratch[4 * static_cast<size_t>(i)] = first;
                a.p.scratch[4 * static_cast<size_t>(i) + 1] = h0;
                a.p.scratch[4 * static_cast<size_t>(i) + 2] = h1;
            }
        }
        __syncthreads();  // wave_tot is free
    }
    if (taken) atomicMax(&taken_s, taken);
    if (bad) atomicOr(&bad_s, bad);
    __syncthreads();
    const int total = carry;  // trim: pages that return
    // Second pass: the new counts (a claim of the call ends; an entry whose slot was claimed before it wrote h0 = h1).
    if (tid == 0) {
        const int now = GROW ? count - taken_s : count + total;
        a.p.state[1] = now < a.p.n_pages ? now : a.p.n_pages;
        if (!FUSED && !GROW) a.p.scratch[4 * static_cast<size_t>(a.p.max_jobs)] = total;
        if (bad_s) atomicOr(reinterpret_cast<uint32_t*>(&a.p.state[0]), bad_s);
    }
    for (int base = 0; base < a.n; base += kScan) {
        const int i = base + tid;
        if (i >= a.n) break;
        const int32_t s = a.slots[i];
        if (s < 0 || s >= a.p.max_jobs) continue;
        const int h0 = FUSED ? sh_h0[i] : a.p.scratch[4 * static_cast<size_t>(i) + 1];
        const int h1 = FUSED ? sh_h1[i] : a.p.scratch[4 * static_cast<size_t>(i) + 2];
        if (h1 != h0) a.p.held[s] = h1;
        else atomicAnd(&a.p.held[s], ~kClaim);
    }
    if constexpr (FUSED) {
        for (int i = wid; i < a.n; i += kW)
            pages_fill<GROW>(a, i, sh_slot[i], sh_first[i] + (GROW ? 0 : total), sh_h0[i], sh_h1[i], lane, kWave);
    }
}

template <bool GROW>
__global__ __launch_bounds__(kFill) void pages_fill_kernel(FillArgs a, int parts) {
    const int i = blockIdx.x / parts, part = blockIdx.x - i * parts;
    const int32_t* e = a.p.scratch + 4 * static_cast<size_t>(i);
    const int first = e[0] + (GROW ? 0 : a.p.scratch[4 * static_cast<size_t>(a.p.max_jobs)]);
    pages_fill<GROW>(a, i, a.slots[i], first, e[1], e[2], part * kFill + threadIdx.x, parts * kFill);
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
    if (a.n <= 128 && work <= 32768)
        return launch_kernel(pages_scan_kernel<GROW, true>, dim3(1), dim3(kScan), 0, st, a);
    ELIS_TRY(launch_kernel(pages_scan_kernel<GROW, false>, dim3(1), dim3(kScan), 0, st, a));
    long long parts = work / (static_cast<long long>(a.n) * 4 * kFill);  // about four elements a thread
    parts = parts < 1 ? 1 : parts > 64 ? 64 : parts;
    if (parts * a.n > 65536) parts = 1;
    return launch_kernel(pages_fill_kernel<GROW>, dim3(static_cast<unsigned>(parts * a.n)), dim3(kFill), 0, st, a, static_cast<int>(parts));
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
