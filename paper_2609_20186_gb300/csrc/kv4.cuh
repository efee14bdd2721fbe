// kv4.cuh -- the 4-bit paged cache: its layout, and checks that the operators on it share.
//
// A (page, head) of a cache of P tokens a page and D = 64 G dimensions is one run of bytes:
//     key codes    [P][D / 8] words     word c * 2G + 2g + i holds dimensions 64 g + 16 c + 8 i + 0 .. 7 of a token
//     value codes  [P / 8][D] words     the word of a dimension holds eight tokens
//     scales       [P][2 G] f16         the key's, then the value's
// Element j = 2 p + e of a word is its nibble p + 4 e, so that one mask takes a pair (2 p, 2 p + 1) to the low bits of
// the word's two halves.  Why this layout: the attention's matrix instructions take a pair of neighbours along the
// contracted axis in one register -- dimensions for the keys, tokens for the values --, and one 16-byte load then
// brings a thread its own elements of both groups of a key, or of four dimensions of a value block, with no exchange
// between threads.  One scale per 64 dimensions lets the keys' scales be applied to the scores and the values' to the
// softmax's weights, so that no unpacked value is multiplied on its own.  Its 7 significant bits make
// (code - 8) * scale an f16 number, so that what the cache holds does not depend on how it is read.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "switchsd_target.h"

namespace switchsd {

constexpr float kScaleMax = 8128.f;  // 127 * 64: the largest 7-bit scale with 8 * scale in f16's range

inline bool kv4_page_ok(int32_t page) {
    return page >= 16 && page <= 256 && (page & (page - 1)) == 0;
}
inline bool kv4_dim_ok(int32_t D) { return D == 64 || D == 128; }
__host__ __device__ inline constexpr int kv4_page_bytes(int page, int D) { return page * (D + (D / 64) * 4); }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
// A stride of a dimension of n: no address goes by that of a dimension of one.
inline bool stride_ok(int64_t stride, int32_t n) { return n == 1 || (stride >= 0 && stride % 8 == 0); }
inline int64_t stride_of(int64_t stride, int32_t n) { return n == 1 ? 0 : stride; }
inline int log2_of(int32_t pow2) {
    int s = 0;
    while ((1 << s) < pow2) ++s;
    return s;
}

// Byte offsets inside a (page, head).
template <int D>
struct Kv4 {
    static constexpr int G = D / 64;
    static constexpr int kRow = D / 2;         // bytes of a token's key codes
    static constexpr int kBlock = 4 * D;       // bytes of eight tokens' value codes
    static constexpr int kScales = 4 * G;      // bytes of a token's scales
    __device__ static int values(int page) { return page * kRow; }
    __device__ static int scales(int page) { return page * D; }
};

}  // namespace switchsd
