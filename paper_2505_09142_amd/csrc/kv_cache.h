// The 4-bit KV cache's records, shared by the kernels that write and read them.
//
// A page holds, for every kv head, page_tokens / 16 records of 16 tokens. A record of d_head D has 17 D bytes:
//   keys    [16][D / 2]           E2M1 pairs, value 2m in the low half of byte m
//   values  [4][16][4][D / 32]    token 4a + b, column c: values (D / 16) c .. (D / 16)(c + 1) - 1 at [a][c][b]
//   scales  keys [16][D / 32], values [4][D / 32][4]   E8M0: 2^(byte - 127), one for 32 values; 255 is NaN
// With the values interleaved by four tokens, the 16 bytes (D 64: 8) a lane loads are its V^T operand's rows for four
// keys, and the 4 scale bytes beside them the scales of exactly those keys.
#pragma once

#include "kernels.h"

namespace elis {

template <int D>
struct Rec {
    static constexpr int kGroups = D / 32;
    static constexpr int kValues = 8 * D;           // byte offset of the values
    static constexpr int kScaleK = 16 * D;          // of the keys' scales
    static constexpr int kScaleV = 16 * D + D / 2;  // of the values' scales
    static constexpr int kBytes = 17 * D;
    __device__ static constexpr int key_at(int tok, int byte) { return tok * (D / 2) + byte; }
    __device__ static constexpr int val_at(int tok, int col) { return kValues + ((tok >> 2) * 64 + col * 4 + (tok & 3)) * (D / 32); }
    __device__ static constexpr int scale_k_at(int tok, int g) { return kScaleK + tok * kGroups + g; }
    __device__ static constexpr int scale_v_at(int tok, int g) { return kScaleV + ((tok >> 2) * kGroups + g) * 4 + (tok & 3); }
};

// Record `tile` of kv head h in a page (byte offset from the first page).
__device__ __forceinline__ size_t rec_offset(const KvCacheView& c, int page, int h, int tile) {
    return ((static_cast<size_t>(page) * c.n_kv_heads + h) * (c.page_tokens / kRecTokens) + tile) * (17 * static_cast<size_t>(c.d_head));
}

}  // namespace elis
