// How a call of the cached attention is launched, from its sizes alone (host code), and which rows its join takes.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace elis {

constexpr int kRecTokens = 16;  // tokens of a record of the cache

// Launches of one call: requests of up to `small` rows (new tokens x heads of a group) in one tile of 16 small_nb rows and
// chunks of small_chunk keys, longer ones in tiles of 16 many_nb rows.
struct KvAttnPlan {
    int small, small_nb, small_rows, small_chunk, small_chunks;
    bool once;  // of those, records loaded past the caches
    bool many;
    int many_nb, many_tiles, many_chunk, many_chunks;
    long long small_most, many_most;  // chunks at most, with any window
    size_t small_parts, many_parts;  // chunk results to join (d_head floats and two more each)
};

inline long long kv_round_up(long long x, long long to) { return (x + to - 1) / to * to; }

// Short requests: records at most, from which on they are loaded past the caches. Nobody reads them again in a call, and in
// the next one only what the memory-side cache of 256 MB holds is worth finding there (jobs, their median and longest length,
// 8 kv heads of 128, through and past the caches: 48 of 16,000, 32,768 206 and 183 us; 128 of 1,500, 4,096 63 and 57.5; 90 of
// 1,200, 4,300 38.9 and 35.3; but 32 of 2,000, 4,096 25.2 and 26.8; 64 of 900, 3,872 23.3 and 23.9).
constexpr double kOnceBytes = 320 << 20;

// Short requests: chunks. A work-group needs about 4.5 us whatever its keys and 0.5 us for each 128, and joining costs 4
// us, so up to 1,024 keys are not split. Beyond, there should be a work-group for each of 256 CUs (one request of 30,001
// tokens and 8 kv heads: chunks of 512 / 640 / 1,024 / 1,280 keys 14.3 / 14.9 / 13.4 / 14.1 us), and at least three to a request that is
// as long as max_kv, because the others are shorter (one chunk, three and six of them: 64 requests of up to 3,872 tokens
// 23.9 / 23.1 / 24.1, 90 of up to 9,000 44.8 / 38.8 / 39.3, but 64 of up to 1,900 with 12 heads of 64 15.3 / 18.6 / 20.0: the
// join), but not more than the fill of the machine asks for (48 requests of up to 32,768: 512 / 1,024 / 2,048 242 / 219 /
// 206).
//
// Long requests: tiles of 32 rows, of which a CU runs three at a time, a 128-key round of theirs in 1.5 us; or, with heads
// of 128, of 64 rows, two at a time in 2.05. What counts is how many fills of the 256 CUs they take, at 3 : 4 (tokens of 32
// query and 8 kv heads over 9,000 keys: 512 tokens 32 rows 101 us, 64 rows 118; 1,000 165, 147; 1,500 227, 262; 2,048 290,
// 265), if the tiles have about the same keys and single tokens do not fill the gaps (four prompts of 1,024 tokens with no
// keys before them 63 and 67; prompts of up to 900 beside 8 tokens 168 and 182). They are split over the keys where they do
// not fill the machine (two of 185 tokens of 20 heads over 2,676 keys 42 and 26 us; 100 tokens of 8 heads over 9,000: 62 and
// 21); of more than 1,024 rows only up to half a fill, because joining costs more (of 8 heads over 9,000 keys, half and whole
// fill: 200 tokens 30.5 and 29.0, 500 43.0 and 45.8).
inline KvAttnPlan plan_kv_attention(int n, int total_q, int max_q, int max_kv, int n_heads, int n_kv_heads, int d_head, int window) {
    KvAttnPlan p{};
    const int group = n_heads / n_kv_heads;
    const long long most = static_cast<long long>(max_q) * group;
    // keys that a tile (at most 64 tokens) can see, on whole records
    const long long reach = window > 0 && window < max_kv ? static_cast<long long>(window) + (max_q < 64 ? max_q : 64) + kRecTokens : max_kv;
    const long long keys = reach < max_kv ? reach : max_kv;
    // Chunks of the keys, about `want`; returns how many there can be for these sizes with any window: the workspace
    // does not depend on it.
    auto split = [&](long long want, long long least, long long largest, int* chunk, int* chunks) {
        long long c = keys;
        if (keys > 1024 && want > 1) {
            c = kv_round_up((keys + want - 1) / want, 128);
            c = c < least ? least : c > largest ? largest : c;
        }
        *chunk = static_cast<int>(c < 1 ? 1 : kv_round_up(c, 16));
        *chunks = static_cast<int>(keys > *chunk ? (keys + *chunk - 1) / *chunk : 1);
        if (max_kv <= 1024 || want <= 1) return 1LL;
        const long long by_size = (max_kv + largest - 1) / largest;
        return want > by_size ? want : by_size;
    };
    long long small_most = 1, many_most = 1;
    // one tile of 16 or 32 rows holds a request, or (of longer ones) at least a single token
    const long long fit = most <= 32 ? most : group;
    if (fit <= 32) {
        p.small_nb = fit <= 16 ? 1 : 2;
        p.small = 16 * p.small_nb;
        p.small_rows = static_cast<int>(most < p.small ? most : p.small);
        p.many = most > p.small;
        if (p.many && static_cast<long long>(n) * max_q == total_q) p.small = p.small_rows = 0;  // every request looks long
        const long long per = static_cast<long long>(n) * n_kv_heads, want = (256 + per - 1) / per;
        small_most = split(want < 3 ? 3 : want, 256, 2048, &p.small_chunk, &p.small_chunks);
    } else {
        p.many = true;
    }
    p.once = static_cast<double>(n) * keys * n_kv_heads * 17 / 16 * d_head > kOnceBytes;
    p.many_chunks = 1;
    if (p.many) {
        const long long rows = static_cast<long long>(total_q) * group, longer = rows / (p.small + 1);
        const long long t4 = (rows + 63) / 64 * n_kv_heads, t2 = (rows + 31) / 32 * n_kv_heads;
        const bool alone = p.small_rows == 0 || 4LL * n * n_kv_heads * small_most <= t4, even = max_kv > 2LL * max_q;
        p.many_nb = d_head == 128 && alone && even && 4 * ((t4 + 511) / 512) < 3 * ((t2 + 767) / 768) ? 4 : 2;
        const int tile = 16 * p.many_nb;
        p.many_tiles = static_cast<int>(rows / tile + (longer < n ? longer : n));  // at most: every long request's last tile cut
        const long long per = (rows / tile + 1) * n_kv_heads;
        const long long fill = rows <= 1024 ? 256 : 128;
        many_most = split((fill + per - 1) / per, rows <= 1024 ? 512 : 1024, max_kv, &p.many_chunk, &p.many_chunks);
    }
    p.small_parts = p.small_rows > 0 && small_most > 1 ? static_cast<size_t>(n) * n_kv_heads * p.small_rows * small_most : 0;
    p.many_parts = p.many && many_most > 1 ? static_cast<size_t>(total_q) * n_heads * many_most : 0;
    p.small_most = small_most;
    p.many_most = many_most;
    return p;
}

// At most, with any window, work-groups of a launch (or rows to join: a work-group each).
inline long long kv_attention_work_groups(const KvAttnPlan& p, int n, int n_kv_heads) {
    const long long small = static_cast<long long>(n) * n_kv_heads;
    const long long parts = small * p.small_most + static_cast<long long>(n_kv_heads) * p.many_tiles * p.many_most;
    const long long joins = p.small_most > 1 ? small * p.small_rows : 0;  // rows of long requests are fewer where they are split
    return parts > joins ? parts : joins;
}

// Row of the chunk results that (request, kv head, row) of a short request or (token, head) of a long one has.
__host__ __device__ inline size_t kv_part_row(bool many, int req, int h, int tok, int head, int r, int n_heads, int n_kv_heads, int small_rows) {
    return many ? static_cast<size_t>(tok) * n_heads + head : (static_cast<size_t>(req) * n_kv_heads + h) * small_rows + r;
}

// The launch that joins split rows: `small` rows of short requests (small_rows for each request and kv head), then one for
// each token and head if a long request may be split; `wide`: a work-group a row, else a wave.
struct KvJoins {
    long long small, all;
    bool wide;
};

inline KvJoins kv_joins(const KvAttnPlan& p, int n, int total_q, int n_heads, int n_kv_heads) {
    const bool small = p.small_rows > 0 && p.small_chunks > 1, many = p.many && p.many_tiles > 0 && p.many_chunks > 1;
    KvJoins j{};
    j.small = small ? static_cast<long long>(n_kv_heads) * n * p.small_rows : 0;
    j.all = j.small + (many ? static_cast<long long>(total_q) * n_heads : 0);
    j.wide = (small && p.small_chunks > 8) || (many && p.many_chunks > 8);
    return j;
}

// What wave w of it joins; any = false past the last row: a launch has waves in fours.
struct KvJoinRow {
    bool any, many;
    int req, h, r;    // of a short request
    int tok, head;    // of a long one
};

__host__ __device__ inline KvJoinRow kv_join_row(long long w, const KvJoins& j, int small_rows, int n_heads, int n_kv_heads) {
    KvJoinRow x{};
    x.any = w < j.all;
    x.many = w >= j.small;
    if (x.many) {
        w -= j.small;
        x.tok = static_cast<int>(w / n_heads);
        x.head = static_cast<int>(w - static_cast<long long>(x.tok) * n_heads);
    } else {
        x.r = static_cast<int>(w % small_rows);
        const long long u = w / small_rows;
        x.h = static_cast<int>(u % n_kv_heads);
        x.req = static_cast<int>(u / n_kv_heads);
    }
    return x;
}

}  // namespace elis
