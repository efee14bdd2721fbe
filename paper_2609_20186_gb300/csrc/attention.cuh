// attention.cuh -- what the kernels of the attention over the 4-bit cache share.
#pragma once

#include <cuda_bf16.h>

#include <algorithm>

#include "kv4.cuh"

namespace switchsd {

constexpr int kAttnMaxCtas = 1024;
constexpr int kJoinParts = 4;     // partial results whose numbers are on their way together
constexpr float kFloor = -3e38f;  // the maximum of nothing: below every score

struct AttnArgs {
    const uint16_t *q;
    int64_t qs[3];
    const uint8_t *cache;
    const int32_t *table, *lens, *new_lens;
    uint16_t *out;
    float *part;        // [2 * CTAs][rows][D + 4]: output, maximum, sum
    int4 *desc;         // [2 * CTAs]: of a partial result: item's row (-1: none), key head, tile of query rows, flags
                        // (kLate: of the CTA, in its first one)
    int32_t *status;
    int32_t B, T, Hq, Hkv, pages, blocks, page_shift, lens_add, new_add, group, dim;
    float scale;
    int32_t give_up;  // attention_tc.cu: a diagnostic, see tc_give_up()
};

// Flags of a partial result: holds the item's first, last unit; a wait of the CTA ran out.
constexpr int kFirst = 1, kLast = 2, kLate = 4;

// A row's lengths, or false where they are bad.
__device__ __forceinline__ bool row_lengths(const AttnArgs &a, int b, int32_t &len, int32_t &nw) {
    const int64_t l = int64_t(__ldcg(a.lens + b)) + a.lens_add, n = int64_t(__ldcg(a.new_lens + b)) + a.new_add;
    const bool ok = l >= 0 && n >= 0 && n <= a.T && l + n <= (int64_t(a.blocks) << a.page_shift);
    len = ok ? int32_t(l) : 0;
    nw = ok ? int32_t(n) : 0;
    return ok;
}

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// A word's four pairs of codes as pairs of f16 numbers c - 8: the code under the exponent of 1024 is 1024 + c (or, four
// bits higher, 1024 + 16 c), and one operation on the pair takes the rest off exactly.
__device__ __forceinline__ uint32_t pair_sub(uint32_t v) {
    uint32_t r;
    asm("add.f16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(0xe408e408u));  // - 1032
    return r;
}
__device__ __forceinline__ uint32_t pair_sub16(uint32_t v) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(v), "r"(0x2c002c00u), "r"(0xd480d480u));  // / 16 - 72
    return r;
}
__device__ __forceinline__ void signed_codes(uint32_t w, uint32_t (&v)[4]) {
    const uint32_t y = w >> 8;
    v[0] = pair_sub((w & 0x000f000fu) | 0x64006400u);
    v[1] = pair_sub16((w & 0x00f000f0u) | 0x64006400u);
    v[2] = pair_sub((y & 0x000f000fu) | 0x64006400u);
    v[3] = pair_sub16((y & 0x00f000f0u) | 0x64006400u);
}

__device__ __forceinline__ uint4 load16(const uint8_t *p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint2 load8(const uint8_t *p) {
    uint2 v;
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t load4(const uint8_t *p) {
    uint32_t v;
    asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}

template <bool F16>
__device__ __forceinline__ float widen1(uint16_t v) {
    return F16 ? __half2float(__ushort_as_half(v)) : bf16_lo(v);
}
template <bool F16>
__device__ __forceinline__ uint32_t narrow2(float a, float b) {
    if (F16) return pack_f16(a, b);
    const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&r);
}

// A CTA's range [u, u_end) of the units of all items -- `unit` keys of a tile of R query rows --, in order of rows, key
// heads and tiles, and the row b that unit u lies in, whose units begin at `base`.  Every CTA adds the lengths up itself.
// Also: statuses (CTA 0), zeros for the query rows of tokens that are not there, and the CTA's partial results marked as
// none.  All threads call it; u >= u_end: nothing to do.
template <int THREADS>
__device__ __forceinline__ void deal_units(const AttnArgs &a, int R, int unit, int cta, int ctas, int64_t *s_pre /* [THREADS + 2] */, int64_t &u,
                                           int64_t &u_end, int &b, int64_t &base) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int kWarps = THREADS / kWarp;
    const int per = (a.B + THREADS - 1) / THREADS;  // rows of a thread
    auto units_of = [&](int row) -> int64_t {
        int32_t len, nw;
        const bool ok = row_lengths(a, row, len, nw);
        if (a.status && cta == 0) a.status[row] = ok ? SWITCHSD_ROW_OK : SWITCHSD_ROW_BAD_LEN;
        const int64_t tiles = (int64_t(nw) * a.group + R - 1) / R;
        return nw ? tiles * a.Hkv * ((int64_t(len) + nw + unit - 1) / unit) : 0;
    };
    int64_t mine = 0;
    for (int i = 0; i < per; ++i)
        if (tid * per + i < a.B) mine += units_of(tid * per + i);
    int64_t x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(kFull, x, o);
        if (lane >= o) x += y;
    }
    s_pre[tid + 1] = x;
    __syncthreads();
    int64_t add = 0;
    for (int w = 0; w < warp; ++w) add += s_pre[32 * w + 32];
    __syncthreads();
    s_pre[tid + 1] = x + add;
    if (tid == 0) s_pre[0] = 0;
    __syncthreads();
    const int64_t total = s_pre[THREADS];
    const int64_t takers = min(total, int64_t(ctas));  // CTAs with a range: at least one unit each
    u = cta < takers ? total * cta / takers : total;
    u_end = cta < takers ? total * (cta + 1) / takers : total;
    const int row16 = a.Hq * a.dim / 8;  // 16-byte pieces of a token's output
    for (int64_t i = int64_t(warp) * ctas + cta; i < int64_t(a.B) * a.T; i += int64_t(ctas) * kWarps) {
        int32_t len, nw;
        row_lengths(a, int(i / a.T), len, nw);
        if (int(i % a.T) < nw) continue;
        uint4 *o = reinterpret_cast<uint4 *>(a.out) + size_t(i) * row16;
        for (int e = lane; e < row16; e += kWarp) o[e] = make_uint4(0, 0, 0, 0);
    }
    if (tid < 2) a.desc[2 * cta + tid] = make_int4(-1, 0, 0, 0);
    const bool here = u < u_end && u >= s_pre[tid] && u < s_pre[tid + 1];
    int row = 0;
    int64_t at = 0;
    if (here) {
        at = s_pre[tid];
        for (row = tid * per;; ++row) {
            const int64_t n = units_of(row);
            if (u < at + n) break;
            at += n;
        }
    }
    __syncthreads();
    if (here) {
        s_pre[0] = row;
        s_pre[1] = at;
    }
    __syncthreads();
    b = int(s_pre[0]);
    base = s_pre[1];
}

template <bool F16>
__device__ __forceinline__ uint16_t narrow1(float a) {
    return F16 ? __half_as_ushort(__float2half_rn(a)) : __bfloat16_as_ushort(__float2bfloat16_rn(a));
}

// Joins the partial results of the items that several CTAs hold, and writes the statuses of a launch that a CTA gave up
// (here, behind all of its CTAs: the first of them writes the others, at a time of its own).  The join: CTAs (i, .) look after the item whose first part is the
// i-th CTA's, a CTA a query row and a thread a dimension, adding the parts in order.  R query rows a tile.  What bounds it:
// latency, so the parts' number comes from their flags 32 at a time and their numbers kJoinParts at a time (one after the
// other, with 16 CTAs for an item's rows, 68 rows of 17 parts each took 50 us with their attention; now 21 us).  CTAs of
// 128 threads and 32 registers fit beside the attention's last ones; wider ones did not and cost 10 us of 280.
template <bool F16, int D>
__global__ void __launch_bounds__(D, 2048 / D) attn_join_kernel(const AttnArgs a, int R) {
    const int i = blockIdx.x, d = threadIdx.x, lane = threadIdx.x & 31, ctas = int(gridDim.x);
    pdl_wait();
    pdl_trigger();
    int from = 2 * i + 1;
    int4 de = __ldcg(a.desc + from);
    const int4 other = __ldcg(a.desc + 2 * i);
    if ((other.w & kLate) && blockIdx.y == 0 && a.status)
        for (int b = d; b < a.B; b += D) a.status[b] = SWITCHSD_ROW_TIMEOUT;  // some row is not done; which ones, the CTA does not know
    if (de.x < 0 || !(de.w & kFirst)) {
        from = 2 * i;
        de = other;
        if (de.x < 0 || !(de.w & kFirst)) return;
    }
    int n = 1;  // partial results of the item: this CTA's and the next ones' first, up to the one that holds the last unit
    for (int c0 = i + 1; !(de.w & kLast);) {
        const int c = c0 + lane;
        const uint32_t last = __ballot_sync(kFull, c >= ctas || (__ldcg(&a.desc[2 * min(c, ctas - 1)].w) & kLast));
        if (last) {
            n = min(c0 + __ffs(int(last)), ctas) - i;
            break;
        }
        c0 += 32;
    }
    int32_t len, nw;
    row_lengths(a, de.x, len, nw);
    for (int row = int(blockIdx.y); row < R; row += int(gridDim.y)) {
        const int rr = de.z * R + row, t = rr / a.group;
        if (t >= nw) return;
        float mx = kFloor, sum = 0.f, y = 0.f;
        for (int j0 = 0; j0 < n; j0 += kJoinParts) {
            float pm[kJoinParts], ps[kJoinParts], py[kJoinParts], top = mx;
#pragma unroll
            for (int j = 0; j < kJoinParts; ++j) {
                pm[j] = kFloor;
                ps[j] = py[j] = 0.f;
                if (j0 + j < n) {
                    const float *src = a.part + (size_t(j0 + j ? 2 * (i + j0 + j) : from) * R + row) * (D + 4);
                    pm[j] = __ldcg(src + D);
                    ps[j] = __ldcg(src + D + 1);
                    py[j] = __ldcg(src + d);
                }
            }
#pragma unroll
            for (int j = 0; j < kJoinParts; ++j) top = fmaxf(top, pm[j]);
            const float f0 = exp2_approx(mx - top);
            y *= f0;
            sum *= f0;
#pragma unroll
            for (int j = 0; j < kJoinParts; ++j) {
                const float f = exp2_approx(pm[j] - top);
                y = fmaf(py[j], f, y);
                sum = fmaf(ps[j], f, sum);
            }
            mx = top;
        }
        const int h = de.y * a.group + rr - t * a.group;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        a.out[((size_t(de.x) * a.T + t) * a.Hq + h) * D + d] = narrow1<F16>(y * inv);
    }
}

// Joins the partial results of a grid of `ctas`, tiles of R query rows.
template <bool F16, int D>
inline cudaError_t launch_join(const AttnArgs &a, int ctas, int R, cudaStream_t s) {
    const int64_t rows = std::min(int64_t(R), int64_t(a.T) * a.group);
    const unsigned y = unsigned(std::min(int64_t(32), rows));
    return launch_pdl(attn_join_kernel<F16, D>, dim3(unsigned(ctas), y), dim3(D), 0, s, 0u, a, R);
}

// The kernel for many query rows (attention_tc.cu): bytes of partial results, and the launch of it and of its join.
size_t attn_tc_workspace(int D);
cudaError_t launch_attn_tc(AttnArgs a, bool f16, int D, int sms, cudaStream_t s);

}  // namespace switchsd
