// attention_tc.cu -- attention over the 4-bit paged cache for many query rows: the verification of drafts.
//
// Same work, units (128 keys) and partial results as attention.cu, with tiles of 128 query rows, on tcgen05.  One CTA an
// SM, with roles for its warps:
//   1 warp fetches: a unit's key codes, value codes and scales, three bulk copies a page, into a ring of three;
//   4 warps unpack the keys and 4 the values: codes to f16 numbers (c - 8) * scale, which are exact, into shared memory -- K
//     as [key][d] and V transposed as [d][key], both the K-major, 128-byte swizzled form, which the cache's word order gives
//     for one 16-byte store a word --, two stages of each;
//   1 thread issues S = Q K^T (into one of two buffers of tensor memory) and O = P V (P from tensor memory, in S's place);
//   8 warps hold the query rows, two threads a row, half of the keys each: maximum, weights, the weights' sum.
// S of a unit is computed while the weights of the one before it are.  O stays in tensor memory over a CTA's units of an
// item: the weights are taken relative to a maximum that may lag the true one by 2^kTcLag, and only a larger rise makes
// the rows' threads scale O (seldom after the first units).
//
// Numbers: as in attention.cu, but that O's sums over the units are the tensor core's (binary32, truncated): a chain of
// 8 additions a unit.  The weights are 2^11 exp(s - M) in f16, 11 bits down to 2^-25 of the reference; where a unit has
// smaller ones they go into a product of their own, 2^24 higher (kTcLift).  The values' scales are in V here, so a NaN
// among them would reach tokens that do not see it through 0 * NaN: of the new tokens, whose keys not every query row
// sees, a NaN in the value's scale becomes one in the key's, which the mask takes out.
//
// What bounds it: the latencies of the rows' warps, and the instructions of the schedulers that hold the tile's first rows.
// A unit takes about 3,200 cycles -- scores out of tensor memory, the maximum over a row's threads, weights (whose
// exponentials alone are 1,000 cycles of a full tile), weights into tensor memory, a barrier each -- where its two products
// take 500; half of the issue slots and 18 % of the memory's rate are used.  Measured: 64 contexts of 2K to 8K tokens, drafts
// of up to 16, 4 query heads a key head: 256 us; 16 contexts of 8K to 32K, drafts of up to 32, 5 query heads a key head: 274
// us (with the tiles of 16 rows 328 and 611 us).  Where many weights are small, with eight times these queries, they take 420
// and 442 us.  Two numbers an instruction where weights are made and added saved 6 us.  Slower were two groups of row warps on
// units in turn, 16 row warps, one pass over the scores that starts again where the maximum rose, and all of a thread's
// scores loaded together for the weights too (303 us).
#include <algorithm>
#include <cstdlib>

#include "attention.cuh"
#include "tc.cuh"

namespace switchsd {

constexpr int kTcRows = 128;                // query rows of a tile: the MMA's M
constexpr int kTcKeys = 128;                // keys of a unit
constexpr int kSplit = 2;                   // threads of a row
constexpr int kRowWarps = 4 * kSplit, kUnpackWarps = 4;  // (of each: keys, values)
constexpr int kRowThreads = kRowWarps * kWarp, kUnpackThreads = kUnpackWarps * kWarp;
constexpr int kTcThreads = kRowThreads + 2 * kUnpackThreads + 4 * kWarp;
// The last four warps: two without work, then the fetching and the MMAs' one, beside the rows 64 .. 127 on their schedulers,
// which not every tile fills (beside the first rows: 288 us where that took 282).
constexpr int kValueWarp = kRowWarps + kUnpackWarps, kFetchWarp = kValueWarp + kUnpackWarps + 2, kMmaWarp = kFetchWarp + 1;
// Registers a thread of each warpgroup: 640 threads are launched with 96 each, and the shares add up to the same.  (Local
// memory would cost much: little of the L1 is left beside the shared memory.)
constexpr int kRowRegs = 120, kUnpackRegs = 80, kOtherRegs = 80;
static_assert(2 * kRowRegs + 2 * kUnpackRegs + kOtherRegs == 5 * 96, "what one warpgroup gains the others give");
constexpr int kRing = 3;                    // units of codes on their way
constexpr int kBlockBytes = 128 * 128;      // 128 rows of one swizzle row: an operand's 64 elements
constexpr float kTcUp = 11.f;               // log2 of the weight of a score at the reference
constexpr float kTcLag = 4.f;               // log2 of how far a weight may lie above: 2^15 is f16's
constexpr float kTcFar = 4194304.f;         // 2^22: the rounding of references of this size and more would show in the weights
constexpr float kTcSmall = 6.103515625e-5f; // 2^-14
constexpr float kTcLift = 16777216.f;       // 2^24
constexpr int kTcColumns = 512;             // tensor memory: S 2 x 128, O 128, O of the small weights 128

template <int D>
struct TcSmem {
    static constexpr int kQ = (D / 64) * kBlockBytes;    // [D / 64][128 rows][128 bytes]
    static constexpr int kK = (D / 64) * kBlockBytes;    // a stage
    static constexpr int kV = 2 * D * 128;               // a stage: [2 blocks of 64 keys][D rows][128 bytes]
    static constexpr int kRawV = kTcKeys * Kv4<D>::kRow;             // codes of a unit: the keys', then
    static constexpr int kRawS = kRawV + kTcKeys / 8 * Kv4<D>::kBlock;
    static constexpr int kRaw = kRawS + kTcKeys * Kv4<D>::kScales;
    static constexpr int bytes = 1024 + kQ + 2 * (kK + kV) + kRing * kRaw;
};

// A wait that gives up after a number of polls (every one here is for this CTA's own work: some microseconds).  The thread may
// sleep for up to 20 us a poll: a spinning warp takes its scheduler's issue slots from the rows' warps.
__device__ __forceinline__ bool tc_wait(uint64_t *bar, uint32_t parity) {
    const uint32_t addr = smem_addr(bar);
    for (uint32_t it = 0; it < 1u << 15; ++it) {
        uint32_t done;
        asm volatile(
            "{\n"
            ".reg .pred p;\n"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 20000;\n"
            "selp.u32 %0, 1, 0, p;\n"
            "}\n"
            : "=r"(done)
            : "r"(addr), "r"(parity)
            : "memory");
        if (done) return true;
    }
    return false;
}
// The same for all of a warp, whose threads go on together.
__device__ __forceinline__ bool tc_wait_warp(uint64_t *bar, uint32_t parity) { return __all_sync(kFull, tc_wait(bar, parity)); }

// The warps of 32 rows.
__device__ __forceinline__ void rows_barrier(int quarter) { asm volatile("bar.sync %0, %1;\n" ::"r"(1 + quarter), "n"(kSplit * kWarp) : "memory"); }
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float min3(float a, float b, float c) {
    float r;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Two binary32 numbers an instruction.
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 halves_of(uint64_t p) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
    return r;
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// One arrival for a warp, behind all of its threads' work (and their fences).
__device__ __forceinline__ void warp_arrive(uint64_t *bar) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// The eight elements of a word of codes times their scales, of pairs.  (The offset and the scale in one multiply-add, which
// is exact too, wants a second path for the scales whose 72-fold f16 does not have, and was slower.)
__device__ __forceinline__ uint4 scaled_word(uint32_t w, uint4 s) {
    uint32_t y[4];
    signed_codes(w, y);
    return make_uint4(mul_f16x2(y[0], s.x), mul_f16x2(y[1], s.y), mul_f16x2(y[2], s.z), mul_f16x2(y[3], s.w));
}

// The segments of a CTA's range: runs of units of one item.
struct Segment {
    int b, hk, rt;
    int32_t len, nw, first, n, units;
};
struct Segments {
    int b;
    int64_t u, u_end, base;
    __device__ bool next(const AttnArgs &a, Segment &s) {
        while (u < u_end) {
            row_lengths(a, b, s.len, s.nw);
            s.units = (s.len + s.nw + kTcKeys - 1) / kTcKeys;
            const int tiles = s.nw ? (s.nw * a.group + kTcRows - 1) / kTcRows : 0;
            const int64_t all = int64_t(s.units) * tiles * a.Hkv;
            if (u >= base + all) {
                base += all;
                ++b;
                continue;
            }
            const int64_t item = (u - base) / s.units;
            s.first = int32_t((u - base) - item * s.units);
            s.b = b;
            s.hk = int(item / tiles);
            s.rt = int(item % tiles);
            s.n = int32_t(min(int64_t(s.units - s.first), u_end - u));
            u += s.n;
            return true;
        }
        return false;
    }
};

template <bool F16, int D>
__global__ void __launch_bounds__(kTcThreads, 1) attn_tc_kernel(const AttnArgs a) {
    using L = Kv4<D>;
    using S = TcSmem<D>;
    constexpr int G = L::G;
    extern __shared__ uint8_t smem_raw[];
    __shared__ int64_t s_pre[kTcThreads + 2];
    __shared__ __align__(8) uint64_t k_full[2], v_full[2], k_empty[2], v_empty[2], s_full[2], p_full[2], o_full, q_full, stopped, raw_full[kRing], raw_empty[kRing];
    __shared__ uint32_t s_tmem;
    __shared__ uint32_t s_small[2], s_rows[4];         // unit + 1, and segment + 1, that had small weights: of a buffer, of 32 rows
    __shared__ __align__(16) uint32_t s_valid[4][4], s_exist[kRing][4];  // of a unit (mod 4, mod 3): keys that exist and whose page does
    __shared__ Segments s_seg[kRowWarps];              // what a row warp needs again when its segment is done
    __shared__ Segment s_item[kRowWarps];
    __shared__ float s_x[2][kSplit][kTcRows];          // what the threads of a row tell each other, of a unit (mod 2)
    __shared__ __align__(16) uint32_t s_scale[kUnpackWarps][16 * G];  // of the values' warps: scales of pairs of tokens
    __shared__ int s_bad;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int cta = blockIdx.x, ctas = int(gridDim.x);
    uint8_t *base = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    uint8_t *sm_q = base, *sm_k = base + S::kQ, *sm_v = sm_k + 2 * S::kK, *sm_raw = sm_v + 2 * S::kV;

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&k_full[i], kUnpackWarps);
            mbar_init(&v_full[i], kUnpackWarps);
            mbar_init(&k_empty[i], 1);
            mbar_init(&v_empty[i], 1);
            mbar_init(&s_full[i], 2);  // the scores, and the MMA thread: what it has seen of the unpacking warps
            mbar_init(&p_full[i], kRowWarps);
        }
        mbar_init(&o_full, 1);
        mbar_init(&q_full, kRowWarps);
        mbar_init(&stopped, 1);
        for (int i = 0; i < kRing; ++i) {
            mbar_init(&raw_full[i], 1);
            mbar_init(&raw_empty[i], 2 * kUnpackWarps);
        }
        fence_mbar_init();
        s_bad = 0;
        s_small[0] = s_small[1] = 0;
        s_rows[0] = s_rows[1] = s_rows[2] = s_rows[3] = 0;
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_addr(&s_tmem)), "r"(kTcColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    pdl_wait();
    pdl_trigger();
    Segments seg;
    deal_units<kTcThreads>(a, kTcRows, kTcKeys, cta, ctas, s_pre, seg.u, seg.u_end, seg.b, seg.base);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    const int page_mask = (1 << a.page_shift) - 1;
    const size_t head_bytes = size_t(kv4_page_bytes(1 << a.page_shift, D)), page_bytes = head_bytes * a.Hkv;
    const int val_off = L::values(1 << a.page_shift), sc_off = L::scales(1 << a.page_shift);
    // Every wait of this thread has ended in time.  After one that has not, no further wait is begun and no result counts;
    // the row warps still go through their loops, because their barriers want all of them.
    bool ok = !a.give_up || warp == kFetchWarp;
    Segment s;

    if (warp < kRowWarps) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kRowRegs));
        // ------------------------------------------------------------------------------------------- query rows
        const int part = warp >> 2, quarter = warp & 3, row = 32 * quarter + lane;
        constexpr int KT = kTcKeys / kSplit, DT = D / kSplit;  // a thread's keys of a unit, and dimensions
        static_assert(KT % 32 == 0 && DT % 16 == 0, "whole words of keys, whole loads of dimensions");
        const uint32_t lanes = tmem + (uint32_t(32 * quarter) << 16);
        uint32_t i = 0, nseg = 0;  // units and segments so far
        auto of_row = [&](auto op) {  // over what the row's threads have put down
            float x = s_x[i & 1][0][row];
#pragma unroll
            for (int p = 1; p < kSplit; ++p) x = op(x, s_x[i & 1][p][row]);
            return x;
        };
        while (seg.next(a, s)) {
            if (lane == 0) {  // (registers are short)
                s_seg[warp] = seg;
                s_item[warp] = s;
            }
            const int rows = min(kTcRows, s.nw * a.group - s.rt * kTcRows);
            const bool mine = row < rows, warp_mine = 32 * quarter < rows;
            const int rr = s.rt * kTcRows + row, t = rr / a.group, h = s.hk * a.group + rr - t * a.group;
            const int32_t limit = mine ? s.len + t : -1;
            float scale;  // of a sum of products, for the binary logarithm: positive (the sign is in the queries)
            {
                // the thread's part of the query, scaled by the power of two that brings the row's largest into [2^11, 2^12)
                const uint16_t *q = a.q + s.b * a.qs[0] + int64_t(t) * a.qs[1] + int64_t(h) * a.qs[2] + part * DT;
                uint4 raw[DT / 8];
                float big = 0.f;
#pragma unroll
                for (int k = 0; k < DT / 8; ++k) {
                    raw[k] = mine ? *reinterpret_cast<const uint4 *>(q + 8 * k) : make_uint4(0, 0, 0, 0);
                    const uint32_t w[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) big = fmaxf(big, fmaxf(fabsf(widen1<F16>(uint16_t(w[e]))), fabsf(widen1<F16>(uint16_t(w[e] >> 16)))));
                }
                s_x[i & 1][part][row] = big;
                rows_barrier(quarter);
                big = of_row([](float x, float y) { return fmaxf(x, y); });
                int ex = 11 - (int(__float_as_uint(big) >> 23) - 127);
                ex = big > 0.f && big < INFINITY ? max(-100, min(100, ex)) : 0;
                const float up = copysignf(__int_as_float((127 + ex) << 23), a.scale);
                scale = __int_as_float((127 - ex) << 23) * fabsf(a.scale) * 1.4426950408889634f;
                if (scale == 0.f) scale = 1e-37f;  // (-inf * 0 would be NaN)
#pragma unroll
                for (int k = 0; k < DT / 8; ++k) {
                    const uint32_t w[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
                    uint32_t y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = pack_f16(widen1<F16>(uint16_t(w[e])) * up, widen1<F16>(uint16_t(w[e] >> 16)) * up);
                    const int d = part * DT + 8 * k;
                    *reinterpret_cast<uint4 *>(sm_q + (d / 64) * kBlockBytes + row * 128 + ((((d % 64) / 8) ^ (row & 7)) * 16)) = make_uint4(y[0], y[1], y[2], y[3]);
                }
                fence_proxy_async();
                warp_arrive(&q_full);
            }
            float m = kFloor, l = 0.f;
            ++nseg;
            for (int32_t k = 0; k < s.n; ++k, ++i) {
                const int buf = int(i & 1);
                const int32_t key0 = (s.first + k) * kTcKeys;
                ok = ok && tc_wait_warp(&s_full[buf], (i >> 1) & 1);
                tc_fence_after();
                const uint32_t sa = lanes + buf * 128 + part * KT;  // this thread's scores; its weights take their place
                const uint4 valid4 = *reinterpret_cast<const uint4 *>(s_valid[i & 3]);
                const bool masked = key0 + kTcKeys > s.len + 1 || (valid4.x & valid4.y & valid4.z & valid4.w) != 0xffffffffu;
                float top = -INFINITY, low = INFINITY;
                if (warp_mine) {
                    if (masked) {  // -inf in the place of the scores that the row does not see
#pragma unroll 1
                        for (int w = 0; w < KT / 32; ++w) {
                            float v[32];
                            tmem_ld32(sa + 32 * w, v);
                            tmem_wait_ld();
                            const int place = part * KT + 32 * w;
                            const int32_t ahead = limit - (key0 + place);  // the last visible key's place
                            const uint32_t see = s_valid[i & 3][place / 32] & (ahead >= 31 ? 0xffffffffu : ahead < 0 ? 0u : (2u << ahead) - 1u);
                            uint32_t y[16];
#pragma unroll
                            for (int e = 0; e < 32; ++e) {
                                const bool in = (see >> e) & 1;
                                low = in ? fminf(low, v[e]) : low;
                                v[e] = in ? v[e] : -INFINITY;
                                top = fmaxf(top, v[e]);
                                y[e & 15] = __float_as_uint(v[e]);
                                if ((e & 15) == 15) tmem_st16(sa + 32 * w + (e & 16), y);
                            }
                        }
                        tmem_wait_st();
                    } else {
                        float v[KT];  // loaded together: a load's latency is most of what this pass takes
#pragma unroll
                        for (int w = 0; w < KT / 32; ++w) tmem_ld32(sa + 32 * w, v + 32 * w);
                        tmem_wait_ld();
                        float t2[4] = {v[0], v[1], v[2], v[3]}, l2[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
                        for (int e = 4; e < KT; e += 2) {
                            t2[(e >> 1) & 3] = max3(t2[(e >> 1) & 3], v[e], v[e + 1]);
                            l2[(e >> 1) & 3] = min3(l2[(e >> 1) & 3], v[e], v[e + 1]);
                        }
                        top = fmaxf(max3(t2[0], t2[1], t2[2]), t2[3]);
                        low = fminf(min3(l2[0], l2[1], l2[2]), l2[3]);
                    }
                }
                const float mn = low * scale;
                s_x[i & 1][part][row] = fmaxf(kFloor, top * scale);
                rows_barrier(quarter);
                const float mx = of_row([](float x, float y) { return fmaxf(x, y); });
                float corr = 1.f;
                if (mx > m + kTcLag) {
                    corr = exp2_approx(m - mx);
                    m = mx;
                    l *= corr;
                }
                const float off = kTcUp - m;
                if (warp_mine) {
                    if (k > 0 && __any_sync(kFull, corr != 1.f)) {  // the units' sums so far, to the new reference
                        ok = ok && tc_wait_warp(&o_full, (i - 1) & 1);
                        tc_fence_after();
                        const bool lo = s_rows[quarter] == nseg;
#pragma unroll 1
                        for (int e = 0; e < (lo ? 2 * DT : DT); e += 16) {
                            const uint32_t at = lanes + (e < DT ? 256 + e : 384 + e - DT) + part * DT;
                            uint32_t w[16];
                            tmem_ld16(at, w);
                            tmem_wait_ld();
#pragma unroll
                            for (int j = 0; j < 16; ++j) w[j] = __float_as_uint(__uint_as_float(w[j]) * corr);
                            tmem_st16(at, w);
                        }
                    }
                    // Some weight below 2^-14?  Its warp says so, and what rounding to f16 leaves of such weights goes into the
                    // other 16 columns of 32 keys; else zeros do, for another warp's sake.
                    const bool small = __any_sync(kFull, mn + off < -14.f);
                    if (small && lane == 0) {
                        s_small[buf] = i + 1;
                        s_rows[quarter] = nseg;  // (read behind the rows' next barrier)
                    }
                    const uint64_t scale2 = pair_of(scale, scale), off2 = pair_of(off, off);
                    uint64_t sum[2] = {0, 0};
                    auto weigh = [&](auto exponents) {
#pragma unroll 1
                        for (int w = 0; w < KT / 32; ++w) {  // 32 keys: 16 words of weights in the first 16 of their scores' columns
                            float v[32];
                            uint32_t y[16];
                            tmem_ld32(sa + 32 * w, v);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const float2 x = exponents(v[2 * e], v[2 * e + 1]);
                                v[2 * e] = exp2_approx(x.x);
                                v[2 * e + 1] = exp2_approx(x.y);
                                sum[e & 1] = add_pair(sum[e & 1], pair_of(v[2 * e], v[2 * e + 1]));
                                y[e] = pack_f16(v[2 * e], v[2 * e + 1]);
                            }
                            tmem_st16(sa + 32 * w, y);
                            if (small) {
#pragma unroll
                                for (int e = 0; e < 32; ++e) v[e] = v[e] < kTcSmall ? (v[e] - __half2float(__float2half_rn(v[e]))) * kTcLift : 0.f;
#pragma unroll
                                for (int e = 0; e < 16; ++e) y[e] = pack_f16(v[2 * e], v[2 * e + 1]);
                            } else {
#pragma unroll
                                for (int e = 0; e < 16; ++e) y[e] = 0;
                            }
                            tmem_st16(sa + 32 * w + 16, y);
                        }
                    };
                    // (a form of its own for references that large: in one, with what is seldom put in the scores' places first, drafts
                    // took 1 to 5 % more)
                    if (__any_sync(kFull, fabsf(m) > kTcFar && m > kFloor))  // the products rounded as the reference's was
                        weigh([&](float x, float y) { return make_float2(__fsub_rn(__fmul_rn(x, scale), m) + kTcUp, __fsub_rn(__fmul_rn(y, scale), m) + kTcUp); });
                    else
                        weigh([&](float x, float y) { return halves_of(fma_pair(pair_of(x, y), scale2, off2)); });
                    const float2 both = halves_of(add_pair(sum[0], sum[1]));
                    l += both.x + both.y;
                    tmem_wait_st();
                }
                // The product of the unit before, every one in turn and before this warp's arrival, without which the next one
                // does not begin: a barrier tells only neighbouring phases apart.
                if (k > 0) ok = ok && tc_wait_warp(&o_full, (i - 1) & 1);
                tc_fence_before();
                warp_arrive(&p_full[buf]);
            }
            // --- the segment's result ---------------------------------------------------------------------------
            s_x[i & 1][part][row] = l;
            rows_barrier(quarter);
            l = of_row([](float x, float y) { return x + y; });
            ok = ok && tc_wait_warp(&o_full, (i - 1) & 1);
            tc_fence_after();
            seg = s_seg[warp];
            s = s_item[warp];
            const bool lo = s_rows[quarter] == nseg;
            const bool whole = s.first == 0 && s.n == s.units;
            const float inv = l == 0.f ? 0.f : 1.f / l;
            const int slot = 2 * cta + (nseg == 1 ? 0 : 1);
            float *partial = a.part + (size_t(slot) * kTcRows + row) * (D + 4);
            const int rows_now = min(kTcRows, s.nw * a.group - s.rt * kTcRows), r0 = s.rt * kTcRows + row, t0 = r0 / a.group;
            const bool out_mine = row < rows_now;
            uint16_t *out = a.out + ((size_t(s.b) * a.T + t0) * a.Hq + s.hk * a.group + r0 - t0 * a.group) * D;
            if (32 * quarter < rows_now) {
#pragma unroll 1
                for (int e = 0; e < DT; e += 16) {
                    float v[16];
                    uint32_t w[16];
                    const int d = part * DT + e;
                    tmem_ld16(lanes + 256 + d, w);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] = __uint_as_float(w[j]);
                    if (lo) {
                        tmem_ld16(lanes + 384 + d, w);
                        tmem_wait_ld();
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] = fmaf(__uint_as_float(w[j]), 1.f / kTcLift, v[j]);
                    }
                    if (out_mine && whole) {
                        uint4 *dst = reinterpret_cast<uint4 *>(out + d);
#pragma unroll
                        for (int j = 0; j < 16; j += 8)
                            dst[j / 8] = make_uint4(narrow2<F16>(v[j] * inv, v[j + 1] * inv), narrow2<F16>(v[j + 2] * inv, v[j + 3] * inv),
                                                    narrow2<F16>(v[j + 4] * inv, v[j + 5] * inv), narrow2<F16>(v[j + 6] * inv, v[j + 7] * inv));
                    } else if (out_mine) {
#pragma unroll
                        for (int j = 0; j < 16; j += 4) *reinterpret_cast<float4 *>(partial + d + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                    }
                }
            }
            if (!whole && out_mine && part == 0) {
                partial[D] = m;
                partial[D + 1] = l;
                if (row == 0) a.desc[slot] = make_int4(s.b, s.hk, s.rt, (s.first == 0 ? kFirst : 0) | (s.first + s.n == s.units ? kLast : 0));
            }
            tc_fence_before();
            rows_barrier(quarter);  // all threads of a row have read s_x
        }
    } else if (warp < kValueWarp + kUnpackWarps) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kUnpackRegs));
        // ------------------------------------------------------------------------------------------- codes to f16
        const bool of_keys = warp < kValueWarp;
        const int uw = warp & (kUnpackWarps - 1), r = lane >> 2, c = lane & 3;  // this warp's keys of a unit: 32 uw .. + 31
        // The 16 bits of a key's or a value's scale, of the warp's key `place`, group g: zero where the key does not exist; a
        // NaN in the value's scale of a new token goes to its key's.  `plain`: all exist, and none is new.
        auto scale_of = [&](const uint8_t *raw, int place, int g, bool of_value, bool plain, uint32_t exists, int32_t key0, int32_t len) -> uint32_t {
            const uint16_t *x = reinterpret_cast<const uint16_t *>(raw + S::kRawS + (32 * uw + place) * L::kScales);
            const uint32_t it = x[(of_value ? G : 0) + g];
            if (plain) return it;
            bool nan = false;
#pragma unroll
            for (int e = 0; e < G; ++e) nan |= (x[G + e] & 0x7fffu) > 0x7c00u;
            const bool gone = !((exists >> place) & 1), moved = nan && key0 + place > len;
            return gone || (moved && of_value) ? 0u : moved ? 0x7e00u : it;
        };
        auto keys = [&](uint32_t i, int32_t key0, int32_t len) {
            const int st = int(i & 1), rs = int(i % kRing);
            ok = tc_wait_warp(&raw_full[rs], (i / kRing) & 1);
            if (i >= 2) ok = ok && tc_wait_warp(&k_empty[st], ((i >> 1) - 1) & 1);
            if (!ok) return;
            const uint32_t exists = s_exist[rs][uw];
            const bool plain = exists == 0xffffffffu && key0 + 32 <= len + 1;
            const uint8_t *raw = sm_raw + rs * S::kRaw;
            // lane (r, c): words 4 c .. of key 8 j + r; the row's place in its swizzled block does not depend on j
            uint8_t *dk = sm_k + st * S::kK + (32 * uw + r) * 128;
            const int at0 = ((2 * c) ^ r) * 16, at1 = ((2 * c + 1) ^ r) * 16;
#pragma unroll 1
            for (int j = 0; j < 4; ++j, dk += 1024) {  // (a loop: the roles' code has to fit the instruction cache together)
                const uint8_t *src = raw + (32 * uw + 8 * j + r) * L::kRow + 8 * G * c;
                uint32_t kw[2 * G];
                if (G == 2) {
                    const uint4 w = *reinterpret_cast<const uint4 *>(src);
                    kw[0] = w.x;
                    kw[1] = w.y;
                    kw[2 * G - 2] = w.z;
                    kw[2 * G - 1] = w.w;
                } else {
                    const uint2 w = *reinterpret_cast<const uint2 *>(src);
                    kw[0] = w.x;
                    kw[1] = w.y;
                }
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const uint32_t x = scale_of(raw, 8 * j + r, g, false, plain, exists, key0, len), x2 = x | (x << 16);
                    const uint4 k4 = make_uint4(x2, x2, x2, x2);
                    *reinterpret_cast<uint4 *>(dk + g * kBlockBytes + at0) = scaled_word(kw[2 * g], k4);
                    *reinterpret_cast<uint4 *>(dk + g * kBlockBytes + at1) = scaled_word(kw[2 * g + 1], k4);
                }
            }
            warp_arrive(&raw_empty[rs]);
            if (lane == 0) s_valid[i & 3][uw] = exists;  // (unit i + 4's keys come after unit i's weights)
            fence_proxy_async();
            warp_arrive(&k_full[st]);
        };
        auto values = [&](uint32_t i, int32_t key0, int32_t len) {
            const int st = int(i & 1), rs = int(i % kRing);
            ok = tc_wait_warp(&raw_full[rs], (i / kRing) & 1);
            if (i >= 2) ok = ok && tc_wait_warp(&v_empty[st], ((i >> 1) - 1) & 1);
            if (!ok) return;
            const uint32_t exists = s_exist[rs][uw];
            const bool plain = exists == 0xffffffffu && key0 + 32 <= len + 1;
            const uint8_t *raw = sm_raw + rs * S::kRaw;
            // the scales of tokens 2 p and 2 p + 1 of block j, group g, in a word: lane 4 (G j + g) + p makes it
            if (lane < 16 * G) {
                const int j = lane / (4 * G), g = (lane / 4) % G, p = lane & 3;
                s_scale[uw][lane] = scale_of(raw, 8 * j + 2 * p, g, true, plain, exists, key0, len) |
                                    (scale_of(raw, 8 * j + 2 * p + 1, g, true, plain, exists, key0, len) << 16);
            }
            __syncwarp();
            const uint32_t *src = reinterpret_cast<const uint32_t *>(raw + S::kRawV + 4 * uw * L::kBlock) + lane;
            uint8_t *dv = sm_v + st * S::kV + (uw >> 1) * (D * 128) + lane * 128;
#pragma unroll 1
            for (int j = 0; j < 4; ++j, src += L::kBlock / 4) {
                const int at = ((4 * (uw & 1) + j) ^ (lane & 7)) * 16;  // of the block's 16 bytes in dimension lane's row
#pragma unroll
                for (int e = 0; e < D / 32; ++e)
                    *reinterpret_cast<uint4 *>(dv + e * 4096 + at) =
                        scaled_word(src[32 * e], *reinterpret_cast<const uint4 *>(&s_scale[uw][4 * (G * j + e / 2)]));
            }
            warp_arrive(&raw_empty[rs]);
            fence_proxy_async();
            warp_arrive(&v_full[st]);
        };
        uint32_t i = 0;
        while (ok && seg.next(a, s)) {
            for (int32_t k = 0; ok && k < s.n; ++k, ++i) {
                const int32_t key0 = (s.first + k) * kTcKeys + 32 * uw;
                if (of_keys)
                    keys(i, key0, s.len);
                else
                    values(i, key0, s.len);
            }
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kOtherRegs));
        if (warp == kFetchWarp) {
        // ------------------------------------------------------------------------------------------- fetching
        // Lane 3 q + p copies part p (key codes, value codes, scales) of the unit's q-th run of keys inside a page.
        const int run = min(kTcKeys, 1 << a.page_shift), runs = kTcKeys / run;
        const int q = lane / 3, part = lane - 3 * q;
        const uint32_t bytes = uint32_t(run) * (part < 2 ? L::kRow : L::kScales);  // (8 tokens' value codes are 8 rows' bytes)
        const int from = part == 0 ? 0 : part == 1 ? val_off : sc_off, to = part == 0 ? 0 : part == 1 ? S::kRawV : S::kRawS;
        uint32_t i = 0;
        int32_t k = 0, page = -1;
        auto find = [&]() {  // the page of this lane's run in unit k of the segment
            const int32_t key = (s.first + k) * kTcKeys + q * run;
            page = q < runs && key < s.len + s.nw ? __ldcg(a.table + size_t(s.b) * a.blocks + (key >> a.page_shift)) : -1;
        };
        bool more = seg.next(a, s);
        if (more) find();
        while (more) {
            const int rs = int(i % kRing);
            if (i >= kRing) ok = tc_wait_warp(&raw_empty[rs], (i / kRing - 1) & 1);
            if (!ok) break;
            const int32_t key0 = (s.first + k) * kTcKeys, total = s.len + s.nw;
            const bool good = uint32_t(page) < uint32_t(a.pages);
            const uint32_t goods = __ballot_sync(kFull, good);
            // the keys that exist: lane w has word w
            uint32_t word = 0;
            if (lane < 4) {
                for (int x = 0; x < 32; x += 16) {  // runs are multiples of 16 keys
                    const int key = 32 * lane + x;
                    const int left = total - (key0 + key);
                    if ((goods >> (3 * (key / run))) & 1) word |= (left >= 16 ? 0xffffu : left > 0 ? (1u << left) - 1u : 0u) << x;
                }
                s_exist[rs][lane] = word;
            }
            __syncwarp();
            if (lane == 0) {
                const int n = __popc(goods & 0x9249249u);  // runs: every third lane
                mbar_arrive_expect_tx(&raw_full[rs], uint32_t(n * run) * (2 * L::kRow + L::kScales));
            }
            __syncwarp();
            if (good)
                bulk_g2s(sm_raw + rs * S::kRaw + to + q * bytes,
                         a.cache + size_t(s.hk) * head_bytes + size_t(page) * page_bytes + from + uint32_t(key0 & page_mask) / run * bytes, bytes, &raw_full[rs]);
            ++i;
            if (++k == s.n) {
                k = 0;
                more = seg.next(a, s);
            }
            if (more) find();
        }
        // copies in flight write shared memory: it stays the CTA's until they have come (also where another warp gave up on them)
        for (uint32_t j = i > kRing ? i - kRing : 0; j < i; ++j) (void)tc_wait(&raw_full[j % kRing], (j / kRing) & 1);
        } else if (warp == kMmaWarp && lane == 0) {
        // ------------------------------------------------------------------------------------------- the MMAs
        uint32_t i = 0, nseg = 0;
        const uint64_t dq = sw128_desc(smem_addr(sm_q)), dk0 = sw128_desc(smem_addr(sm_k)), dv0 = sw128_desc(smem_addr(sm_v));
        bool fresh = false, lo = false;        // O of the item: nothing added yet, the small weights' product begun
        auto product = [&](uint32_t j) {       // O += P V of unit j
            const int buf = int(j & 1);
            ok = ok && tc_wait(&v_full[buf], (j >> 1) & 1) && tc_wait(&p_full[buf], (j >> 1) & 1);
            if (!ok) return;
            tc_fence_after();
            const uint64_t dv = dv0 + (buf ? uint64_t(S::kV >> 4) : 0);
            // the weights of 32 keys are in 16 columns of their scores' 32, the small ones in the other 16
            auto keys16 = [&](int k) { return dv + uint64_t(((k >> 2) * (D * 128) + (k & 3) * 32) >> 4); };
#pragma unroll
            for (int k = 0; k < kTcKeys / 16; ++k)
                mma_ts(tmem + 256, tmem + buf * 128 + (k >> 1) * 32 + 8 * (k & 1), keys16(k), f16_idesc(D), !fresh || k != 0);
            if (s_small[buf] == j + 1) {
#pragma unroll
                for (int k = 0; k < kTcKeys / 16; ++k)
                    mma_ts(tmem + 384, tmem + buf * 128 + (k >> 1) * 32 + 16 + 8 * (k & 1), keys16(k), f16_idesc(D), lo || k != 0);
                lo = true;
            }
            fresh = false;
            tc_commit(&v_empty[buf]);
            tc_commit(&o_full);
        };
        while (ok && seg.next(a, s)) {
            for (int32_t k = 0; ok && k < s.n; ++k, ++i) {
                const int buf = int(i & 1);
                if (k == 0) {
                    // (the rows' threads write the queries when they have read the last O)
                    ok = ok && tc_wait(&q_full, nseg & 1);
                    fresh = true;
                    lo = false;
                }
                ok = ok && tc_wait(&k_full[buf], (i >> 1) & 1);
                if (!ok) break;
                mbar_arrive(&s_full[buf]);
                tc_fence_after();
                const uint64_t dk = dk0 + (buf ? uint64_t(S::kK >> 4) : 0);
#pragma unroll
                for (int e = 0; e < D / 16; ++e) {
                    const uint64_t step = uint64_t(((e >> 2) * kBlockBytes + (e & 3) * 32) >> 4);
                    mma_ss(tmem + buf * 128, dq + step, dk + step, f16_idesc(kTcKeys), e != 0);
                }
                tc_commit(&s_full[buf]);
                tc_commit(&k_empty[buf]);
                if (k > 0) product(i - 1);
            }
            if (ok) product(i - 1);  // before the next segment is looked up
            ++nseg;
        }
        // what is in flight reads shared and tensor memory (the rows' threads wait for the last product too, unless they gave up)
        tc_commit(&stopped);
        (void)tc_wait(&stopped, 0);
        }
    }
    if (!ok) s_bad = 1;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kMmaWarp)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(kTcColumns) : "memory");
    if (s_bad && tid == 0) a.desc[2 * cta].w |= kLate;  // (the thread that wrote it; the join writes the statuses)
}

// Whether the environment variable SWITCHSD_DIAG_ATTENTION_GIVE_UP is 1 (read once per process).  A diagnostic of the path
// behind a wait that ran out: the rows', the unpacking and the MMAs' warps give up before their first wait, and the fetching
// one once the ring that nobody empties is full and its own wait has run out; the statuses then say SWITCHSD_ROW_TIMEOUT.
static bool tc_give_up() {
    static const bool set = [] {
        const char *v = std::getenv("SWITCHSD_DIAG_ATTENTION_GIVE_UP");
        return v != nullptr && v[0] == '1' && v[1] == '\0';
    }();
    return set;
}

size_t attn_tc_workspace(int D) { return size_t(2 * kAttnMaxCtas) * sizeof(int4) + size_t(2 * 256) * kTcRows * (D + 4) * sizeof(float); }

template <bool F16, int D>
static cudaError_t launch(const AttnArgs &a, int sms, cudaStream_t s) {
    static bool attr_done[64] = {false};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_done[dev]) {
        e = cudaFuncSetAttribute(attn_tc_kernel<F16, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcSmem<D>::bytes);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_done[dev] = true;
    }
    const unsigned ctas = unsigned(std::min(256, sms));
    // an explicit one-CTA cluster: the MMA commit addresses shared::cluster
    e = launch_pdl(attn_tc_kernel<F16, D>, dim3(ctas), dim3(kTcThreads), size_t(TcSmem<D>::bytes), s, 1u, a);
    if (e != cudaSuccess) return e;
    return launch_join<F16, D>(a, int(ctas), kTcRows, s);
}

cudaError_t launch_attn_tc(AttnArgs a, bool f16, int D, int sms, cudaStream_t s) {
    a.give_up = tc_give_up();
    if (f16) return D == 128 ? launch<true, 128>(a, sms, s) : launch<true, 64>(a, sms, s);
    return D == 128 ? launch<false, 128>(a, sms, s) : launch<false, 64>(a, sms, s);
}

}  // namespace switchsd
