// attention.cu -- switchsd_kv4_attention: attention of a step's new tokens over the 4-bit paged cache.
//
// Work.  The query rows of a row and key head -- its new tokens times the query heads that share the key head -- are cut
// into tiles of 8 or 16; an item is one such tile over its row's keys, and its unit of work is 128 keys.  The units of
// all items, in order, are dealt out evenly over a fixed grid (the lengths are on the device; every CTA adds them up
// itself): a CTA takes a contiguous range, which may begin and end inside an item.  An item that one CTA holds whole is
// written out at once; the others leave partial results (maximum, sum, output) that a second kernel joins in order.
//
// Keys and values never leave the registers.  Per 32 keys a warp computes S^T = K Q^T and O^T += V^T W^T with
// m16n8k16 matrix instructions, the 4-bit codes as the A operand.  The keys' are masked out of the cache's words in
// place -- a code c in the low bits of an f16 is the (subnormal) number c 2^-24 --, so that a word of eight codes costs
// five instructions, and their offset of 8 is the accumulators' start (-8 times the query's sum).  The values' become
// signed numbers, four instructions a word more: taking 8 times the weights' sum off afterwards would leave an error of
// that sum's size where the values are small.  The scales are applied outside: to the scores, and to the weights.
//
// Numbers.  Each query is scaled by a power of two of its own so that it is f16 numbers exactly (a bf16 has fewer bits; what
// lies 2^22 below its largest may lose bits, less than the binary32 sums do), and its scores by the inverse; codes, and so
// keys and values, are exact; scores, maxima, sums and the output are binary32.  (The output's sums over the keys are the
// matrix unit's, which truncates: two additions for 32 keys of a warp, a bias below 2^-23 of the sum each.)  The weights
// 2^12 exp(s - M) * scale_v are rounded to f16 (11 bits): M, the reference, is at most 2^kLag below the running maximum of
// the score plus the logarithm of its value's scale, so that the largest weight fits whatever the scales; what rounding
// leaves of weights below 2^-26 of the reference, where f16 has fewer bits, is multiplied apart, 2^24 higher.
//
// Why the weights are f16: the matrix instructions take them so, and what their rounding leaves of every weight, multiplied
// apart too, would double the values' instructions.  It disappears in a bf16 result; an f16 result over 32K to 128K keys is
// 2.9e-4 off (relative to the result, over all of it) where binary32 weights leave it 2.1e-4 off, its own rounding.
//
// What bounds it: the instructions that unpack codes and weigh scores, at 12 warps an SM, about 56 % of the issue slots.
// Measured: 64 contexts of 8K to 32K tokens, 8 key heads of 128 dimensions, 4 query heads each, one token a row: 353 us,
// of which the 1.4 GB of cache need 60 % alone; 4 contexts of 32K to 128K, 8 query heads each: 98 us (54 %); one
// context of 2K: 11 us, with its join.  Where many weights are small (eight times these queries), the first two take 386 and
// 108 us.
#include <algorithm>

#include "attention.cuh"

namespace switchsd {

constexpr int kAttnWarps = 4;
constexpr int kAttnThreads = kAttnWarps * kWarp;
constexpr int kAttnUnit = kAttnWarps * 32;  // keys of a unit: 32 a warp
// As many CTAs an SM as leave a warp its registers (168; 8 query rows: 2 CTAs 453, 3 CTAs 353, 4 CTAs, which spill, 469 us
// for the first figures above; 16 rows of 64 contexts of 8K: 1 CTA 438, 2 CTAs 235, 3 CTAs 545 us).
constexpr int attn_ctas_per_sm(int NT) { return NT == 1 ? 3 : 2; }
constexpr float kWeightLog = 12.f;          // log2 of the weight of a score (with its value's scale) at the reference
constexpr float kLag = 3.f;                 // log2 of how far one may lie above: 2^15 is f16's
constexpr float kSmall = 6.103515625e-5f;   // 2^-14: below it f16 loses bits
constexpr float kLift = 16777216.f;         // 2^24: of the product of what rounding leaves of small weights

__device__ __forceinline__ float log2_approx(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// D = A B + C of m16n8k16, f16 operands, binary32 sums.
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1,
                                         float c0, float c1, float c2, float c3) {
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};\n"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// From shared memory at every use: kept in registers, the queries would leave room for fewer warps.
__device__ __forceinline__ uint4 load_shared(const uint4 *p) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(smem_addr(p)));
    return v;
}

// The codes and scales of a thread's share of 32 keys.
template <int D>
struct Keys {
    static constexpr int G = D / 64;
    uint32_t k[4][2 * G];   // key tile j: words of the thread's token
    uint32_t sc[4][G];      // scales of the thread's token of tile j: keys' then values', f16
    uint32_t v[D / 32][4];  // value words: dimensions 32 i + 4 r + 0 .. 3, tokens of block c
};

template <bool F16, int D, int NT>
__global__ void __launch_bounds__(kAttnThreads, attn_ctas_per_sm(NT)) attn_kernel(const AttnArgs a) {
    using L = Kv4<D>;
    constexpr int G = L::G, R = 8 * NT, MT = D / 16;  // groups, query rows of a tile, output tiles of 16 dimensions
    extern __shared__ float s_out[];                  // [warps][R][D + 4]
    __shared__ float s_max[kAttnWarps][R], s_sum[kAttnWarps][R];
    __shared__ uint4 s_q[NT][G][2][kWarp];            // queries: B operands of each lane, the same for all warps
    __shared__ int64_t s_pre[kAttnThreads + 2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int r = lane >> 2, c = lane & 3;
    const int cta = blockIdx.x, ctas = int(gridDim.x);
    pdl_wait();
    pdl_trigger();

    int b;
    int64_t u, u_end, base_u;
    deal_units<kAttnThreads>(a, R, kAttnUnit, cta, ctas, s_pre, u, u_end, b, base_u);
    if (u >= u_end) return;
    const int64_t u_begin = u;
    const int page_mask = (1 << a.page_shift) - 1;
    const size_t head_bytes = size_t(kv4_page_bytes(1 << a.page_shift, D));
    const int val_off = L::values(1 << a.page_shift), sc_off = L::scales(1 << a.page_shift);

    while (u < u_end) {
        // --- the item -------------------------------------------------------------------------------------------
        int32_t len, nw;
        row_lengths(a, b, len, nw);
        const int32_t total_keys = len + nw;
        const int32_t units = (total_keys + kAttnUnit - 1) / kAttnUnit;
        const int tiles = nw ? (nw * a.group + R - 1) / R : 0;
        if (u >= base_u + int64_t(units) * tiles * a.Hkv) {  // the next row
            base_u += int64_t(units) * tiles * a.Hkv;
            ++b;
            continue;
        }
        const int64_t item = (u - base_u) / units;
        const int32_t first = int32_t((u - base_u) - item * units);
        const int hk = int(item / tiles), rt = int(item % tiles);
        const int32_t n = int32_t(min(int64_t(units - first), u_end - u));
        const int rows = min(R, nw * a.group - rt * R);

        // --- queries: B operand, row n = lane / 4 of each of NT tiles of 8 --------------------------------------
        float start[NT][G][2];      // -8 sum of the query's group, of columns 2 c, 2 c + 1
        float score[NT][2];         // of the column's query: the binary logarithm's scale of a sum of products
        int32_t limit[NT][2];       // last key that the column's query sees
        {
            uint4 raw[NT][G][2];
            float up[NT];           // of row r's query
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float big = 0.f;
                const int row = 8 * nt + r, rr = rt * R + row, t = rr / a.group, h = hk * a.group + rr - t * a.group;
                const uint16_t *q = a.q + b * a.qs[0] + t * a.qs[1] + h * a.qs[2] + 16 * c;
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        raw[nt][g][i] = row < rows ? *reinterpret_cast<const uint4 *>(q + 64 * g + 8 * i) : make_uint4(0, 0, 0, 0);
                        const uint32_t w[4] = {raw[nt][g][i].x, raw[nt][g][i].y, raw[nt][g][i].z, raw[nt][g][i].w};
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            big = fmaxf(big, fmaxf(fabsf(widen1<F16>(uint16_t(w[e]))), fabsf(widen1<F16>(uint16_t(w[e] >> 16)))));
                    }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row_c = 8 * nt + 2 * c + e;
                    limit[nt][e] = row_c < rows ? len + (rt * R + row_c) / a.group : -1;
                }
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) big = fmaxf(big, __shfl_xor_sync(kFull, big, o));  // a row's four lanes
                // the power of two that brings the row's largest into [2^11, 2^12)
                int ex = 11 - (int(__float_as_uint(big) >> 23) - 127);
                ex = big > 0.f && big < INFINITY ? max(-100, min(100, ex)) : 0;
                up[nt] = __int_as_float((127 + ex) << 23);
                const float down = __int_as_float((127 - ex) << 23) * a.scale * 1.4426950408889634f * 16777216.f;
                score[nt][0] = __shfl_sync(kFull, down, 8 * c);
                score[nt][1] = __shfl_sync(kFull, down, 8 * c + 4);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    float sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t w[4] = {raw[nt][g][i].x, raw[nt][g][i].y, raw[nt][g][i].z, raw[nt][g][i].w};
                        uint32_t qb[4];            // [step x register]
#pragma unroll
                        for (int e = 0; e < 4; ++e) {  // pair e; the odd pairs' codes stand four bits higher
                            const float x0 = widen1<F16>(uint16_t(w[e])) * up[nt], x1 = widen1<F16>(uint16_t(w[e] >> 16)) * up[nt];
                            sum += x0 + x1;
                            const float f = e & 1 ? 0.0625f : 1.f;
                            qb[e] = pack_f16(x0 * f, x1 * f);
                        }
                        if (warp == 0) s_q[nt][g][i][lane] = make_uint4(qb[0], qb[1], qb[2], qb[3]);
                    }
                    sum += __shfl_xor_sync(kFull, sum, 1);
                    sum += __shfl_xor_sync(kFull, sum, 2);
                    start[nt][g][0] = __shfl_sync(kFull, sum, 8 * c) * (-8.f / 16777216.f);
                    start[nt][g][1] = __shfl_sync(kFull, sum, 8 * c + 4) * (-8.f / 16777216.f);
                }
        }
        __syncthreads();  // (every item ends with one too, behind which the next one's queries are written)

        float o[NT][MT][4], m[NT][2], l[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][i][e] = 0.f;
            m[nt][0] = m[nt][1] = kFloor;
            l[nt][0] = l[nt][1] = 0.f;
        }

        // --- the keys, 32 at a time -----------------------------------------------------------------------------
        const int32_t *table = a.table + size_t(b) * a.blocks;
        const uint8_t *cache = a.cache + size_t(hk) * head_bytes;
        const size_t page_bytes = head_bytes * a.Hkv;
        Keys<D> x;
        // groups of eight keys that this thread reads: its keys' token lies in group r / 2, its values' in group c
        auto page_at = [&](int32_t key) -> int32_t {
            return key < total_keys ? __ldcg(table + (key >> a.page_shift)) : -1;
        };
        auto load_keys = [&](int32_t key0, int32_t page) {  // key0: of the 32; page: of group r / 2
            const int32_t at = key0 + 8 * (r >> 1);
            if (uint32_t(page) < uint32_t(a.pages)) {
                const int in = (at & page_mask) + (r & 1);
                const uint8_t *p = cache + size_t(page) * page_bytes;
                const uint8_t *pk = p + in * L::kRow + c * (8 * G), *ps = p + sc_off + in * L::kScales;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (G == 2) {
                        const uint4 w = load16(pk + 2 * j * L::kRow);
                        x.k[j][0] = w.x;
                        x.k[j][1] = w.y;
                        x.k[j][2 * G - 2] = w.z;
                        x.k[j][2 * G - 1] = w.w;
                        const uint2 s = load8(ps + 2 * j * L::kScales);
                        x.sc[j][0] = s.x;
                        x.sc[j][G - 1] = s.y;
                    } else {
                        const uint2 w = load8(pk + 2 * j * L::kRow);
                        x.k[j][0] = w.x;
                        x.k[j][1] = w.y;
                        x.sc[j][0] = load4(ps + 2 * j * L::kScales);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
#pragma unroll
                    for (int i = 0; i < 2 * G; ++i) x.k[j][i] = 0;
#pragma unroll
                    for (int i = 0; i < G; ++i) x.sc[j][i] = 0;
                }
            }
        };
        auto load_values = [&](int32_t key0, int32_t page) {  // page: of group c
            const int32_t at = key0 + 8 * c;
            if (uint32_t(page) < uint32_t(a.pages)) {
                const uint8_t *p = cache + size_t(page) * page_bytes + val_off + ((at & page_mask) >> 3) * L::kBlock + 16 * r;
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const uint4 w = load16(p + 128 * i);
                    x.v[i][0] = w.x;
                    x.v[i][1] = w.y;
                    x.v[i][2] = w.z;
                    x.v[i][3] = w.w;
                }
            } else {
#pragma unroll
                for (int i = 0; i < D / 32; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x.v[i][e] = 0;
            }
        };
        int32_t key0 = first * kAttnUnit + 32 * warp;
        const int32_t key_end = min(total_keys, (first + n) * kAttnUnit);
        int32_t pk = page_at(key0 + 8 * (r >> 1)), pv = page_at(key0 + 8 * c);
        load_keys(key0, pk);
        load_values(key0, pv);
        int32_t pk1 = page_at(key0 + kAttnUnit + 8 * (r >> 1)), pv1 = page_at(key0 + kAttnUnit + 8 * c);
        for (; key0 < key_end; key0 += kAttnUnit) {
            const bool more = key0 + kAttnUnit < key_end;
            const bool out_of_pool = uint32_t(pk) >= uint32_t(a.pages);
            // S^T: tile j (rows r of two matrix tiles) holds keys key0 + 8 (r / 2) + 2 j + r % 2
            float s[NT][4][2];
            float ks[4][G];
            uint32_t value_scales[4];  // (the next keys' scales are loaded before they are used)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                // scales of the token: G of the key, G of the value
                const float2 k2 = __half22float2(*reinterpret_cast<const __half2 *>(&x.sc[j][0]));
                ks[j][0] = k2.x;
                if (G == 2) ks[j][G - 1] = k2.y;
                value_scales[j] = x.sc[j][G - 1];
            }
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        float acc[4];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t w0 = x.k[2 * mt][2 * g + i], w1 = x.k[2 * mt + 1][2 * g + i];
                            const uint4 qb = load_shared(&s_q[nt][g][i][lane]);
                            if (i == 0)
                                mma16816(acc, w0 & 0x000f000fu, w1 & 0x000f000fu, w0 & 0x00f000f0u, w1 & 0x00f000f0u, qb.x, qb.y,
                                         start[nt][g][0], start[nt][g][1], start[nt][g][0], start[nt][g][1]);
                            else
                                mma16816(acc, w0 & 0x000f000fu, w1 & 0x000f000fu, w0 & 0x00f000f0u, w1 & 0x00f000f0u, qb.x, qb.y,
                                         acc[0], acc[1], acc[2], acc[3]);
                            const uint32_t x0 = w0 >> 8, x1 = w1 >> 8;
                            mma16816(acc, x0 & 0x000f000fu, x1 & 0x000f000fu, x0 & 0x00f000f0u, x1 & 0x00f000f0u, qb.z, qb.w,
                                     acc[0], acc[1], acc[2], acc[3]);
                        }
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            if (g == 0) {
                                s[nt][2 * mt][e] = acc[e] * ks[2 * mt][0];
                                s[nt][2 * mt + 1][e] = acc[2 + e] * ks[2 * mt + 1][0];
                            } else {
                                s[nt][2 * mt][e] = fmaf(acc[e], ks[2 * mt][g], s[nt][2 * mt][e]);
                                s[nt][2 * mt + 1][e] = fmaf(acc[2 + e], ks[2 * mt + 1][g], s[nt][2 * mt + 1][e]);
                            }
                            if (g == G - 1) {
                                s[nt][2 * mt][e] *= score[nt][e];
                                s[nt][2 * mt + 1][e] *= score[nt][e];
                            }
                        }
                    }
                }
            if (more) load_keys(key0 + kAttnUnit, pk1);
            // keys that some query of the tile does not see: past its token, past the row's end, or without a page
            const bool masked = __any_sync(kFull, out_of_pool) || key0 + 32 > len + 1;
            if (masked) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int32_t key = key0 + 8 * (r >> 1) + 2 * j + (r & 1);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if (out_of_pool || key > limit[nt][e]) s[nt][j][e] = -INFINITY;
                }
            }
            // Weights: the softmax's times the values' scales.
            float vs[4][G], lg[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 v2 = __half22float2(*reinterpret_cast<const __half2 *>(&value_scales[j]));
                vs[j][0] = G == 2 ? v2.x : v2.y;
                vs[j][G - 1] = v2.y;
                lg[j] = fmaxf(log2_approx(G == 2 ? fmaxf(v2.x, v2.y) : v2.y), -24.f);
            }
            // The reference m may lag the largest score and scale by 2^kLag; only where one lies further above do the columns
            // find their maxima and bring O to the new reference.
            bool beyond = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    beyond |= fmaxf(fmaxf(s[nt][0][e] + lg[0], s[nt][1][e] + lg[1]), fmaxf(s[nt][2][e] + lg[2], s[nt][3][e] + lg[3])) > m[nt][e] + kLag;
            if (__any_sync(kFull, beyond)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float corr[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = fmaxf(fmaxf(s[nt][0][e] + lg[0], s[nt][1][e] + lg[1]), fmaxf(s[nt][2][e] + lg[2], s[nt][3][e] + lg[3]));
#pragma unroll
                        for (int sh = 4; sh < 32; sh <<= 1) mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, sh));
                        mx = fmaxf(mx, m[nt][e]);
                        corr[e] = exp2_approx(m[nt][e] - mx);
                        m[nt][e] = mx;
                        l[nt][e] *= corr[e];
                    }
#pragma unroll
                    for (int i = 0; i < MT; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[nt][i][e] *= corr[e & 1];
                }
            }
            uint32_t wb[NT][G][4];  // transposed: B operand of tile j
            float least = INFINITY;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    // (rounded down: to nearest, a reference from 2^26 on, whose neighbours are 8 and more apart, would let
                    // weights through that f16 does not have)
                    const float off = __fsub_rd(kWeightLog, m[nt][e]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s[nt][j][e] = exp2_approx(s[nt][j][e] + off);
                        l[nt][e] += s[nt][j][e];
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        float w0 = s[nt][j][0] * vs[j][g], w1 = s[nt][j][1] * vs[j][g];
                        if (masked) {  // a scale that a masked key left may be anything
                            w0 = s[nt][j][0] > 0.f ? w0 : 0.f;
                            w1 = s[nt][j][1] > 0.f ? w1 : 0.f;
                            least = fminf(least, fminf(w0 > 0.f ? w0 : INFINITY, w1 > 0.f ? w1 : INFINITY));
                        } else {
                            least = fminf(least, fminf(w0, w1));
                        }
                        wb[nt][g][j] = transpose8x8(pack_f16(w0, w1));
                    }
            }
            // f16 keeps 11 bits down to 2^-14; what rounding leaves of smaller weights is multiplied apart, 2^24 higher
            uint32_t wl[NT][G][4];
            const bool small = __any_sync(kFull, least < kSmall);
            if (small) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int g = 0; g < G; ++g) {
                            float w[2];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float p = s[nt][j][e], y = p * vs[j][g];
                                w[e] = p > 0.f && y < kSmall ? (y - __half2float(__float2half_rn(y))) * kLift : 0.f;
                            }
                            wl[nt][g][j] = transpose8x8(pack_f16(w[0], w[1]));
                        }
            }
            // O^T: the values' codes as signed f16 numbers
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t va[4], vb[4];
                    signed_codes(x.v[i][2 * h], va);
                    signed_codes(x.v[i][2 * h + 1], vb);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const uint32_t(&w)[4] = wb[nt][i / 2];  // (two i a group)
                        float(&oo)[4] = o[nt][2 * i + h];
                        mma16816(oo, va[0], vb[0], va[1], vb[1], w[0], w[1], oo[0], oo[1], oo[2], oo[3]);
                        mma16816(oo, va[2], vb[2], va[3], vb[3], w[2], w[3], oo[0], oo[1], oo[2], oo[3]);
                        if (small) {
                            const uint32_t(&z)[4] = wl[nt][i / 2];
                            float acc[4];
                            mma16816(acc, va[0], vb[0], va[1], vb[1], z[0], z[1], 0.f, 0.f, 0.f, 0.f);
                            mma16816(acc, va[2], vb[2], va[3], vb[3], z[2], z[3], acc[0], acc[1], acc[2], acc[3]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) oo[e] = fmaf(acc[e], 1.f / kLift, oo[e]);
                        }
                    }
                }
            if (more) load_values(key0 + kAttnUnit, pv1);
            pk = pk1;
            pv = pv1;
            pk1 = page_at(key0 + 2 * kAttnUnit + 8 * (r >> 1));
            pv1 = page_at(key0 + 2 * kAttnUnit + 8 * c);
        }

        // --- the four warps' results joined ---------------------------------------------------------------------
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int sh = 4; sh < 32; sh <<= 1) l[nt][e] += __shfl_xor_sync(kFull, l[nt][e], sh);
                const int row = 8 * nt + 2 * c + e;
                if (r == 0) {
                    s_max[warp][row] = m[nt][e];
                    s_sum[warp][row] = l[nt][e];
                }
                float *dst = s_out + (size_t(warp) * R + row) * (D + 4);
#pragma unroll
                for (int i = 0; i < D / 32; ++i)
                    *reinterpret_cast<float4 *>(dst + 32 * i + 4 * r) =
                        make_float4(o[nt][2 * i][e], o[nt][2 * i][2 + e], o[nt][2 * i + 1][e], o[nt][2 * i + 1][2 + e]);
            }
        __syncthreads();
        const bool whole = first == 0 && n == units;
        const int slot = 2 * cta + (u == u_begin ? 0 : 1);
        for (int i = tid; i < R * (D / 4); i += kAttnThreads) {
            const int row = i / (D / 4), d = 4 * (i % (D / 4));
            float mx = kFloor;
#pragma unroll
            for (int w = 0; w < kAttnWarps; ++w) mx = fmaxf(mx, s_max[w][row]);
            float sum = 0.f;
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kAttnWarps; ++w) {
                const float f = exp2_approx(s_max[w][row] - mx);
                const float4 z = *reinterpret_cast<const float4 *>(s_out + (size_t(w) * R + row) * (D + 4) + d);
                sum = fmaf(s_sum[w][row], f, sum);
                y.x = fmaf(z.x, f, y.x);
                y.y = fmaf(z.y, f, y.y);
                y.z = fmaf(z.z, f, y.z);
                y.w = fmaf(z.w, f, y.w);
            }
            if (whole) {
                if (row < rows) {
                    const int rr = rt * R + row, t = rr / a.group, h = hk * a.group + rr - t * a.group;
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    uint2 w = make_uint2(narrow2<F16>(y.x * inv, y.y * inv), narrow2<F16>(y.z * inv, y.w * inv));
                    *reinterpret_cast<uint2 *>(a.out + ((size_t(b) * a.T + t) * a.Hq + h) * D + d) = w;
                }
            } else {
                float *dst = a.part + (size_t(slot) * R + row) * (D + 4);
                *reinterpret_cast<float4 *>(dst + d) = y;
                if (d == 0) {
                    dst[D] = mx;
                    dst[D + 1] = sum;
                }
            }
        }
        if (!whole && tid == 0)
            a.desc[slot] = make_int4(b, hk, rt, (first == 0 ? kFirst : 0) | (first + n == units ? kLast : 0));
        __syncthreads();
        u += n;
    }
}

static size_t attn_workspace(int D, int NT) {
    return std::max(size_t(2 * kAttnMaxCtas) * (sizeof(int4) + size_t(8 * NT) * (D + 4) * sizeof(float)), attn_tc_workspace(D));
}

template <bool F16, int D, int NT>
static cudaError_t launch_attn(AttnArgs a, int sms, cudaStream_t s) {
    static bool attr_done[64] = {false};
    const size_t smem = size_t(kAttnWarps) * 8 * NT * (D + 4) * sizeof(float);
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_done[dev]) {
        e = cudaFuncSetAttribute(attn_kernel<F16, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_done[dev] = true;
    }
    const unsigned ctas = unsigned(std::min(kAttnMaxCtas, sms * attn_ctas_per_sm(NT)));
    e = launch_pdl(attn_kernel<F16, D, NT>, dim3(ctas), dim3(kAttnThreads), smem, s, 0u, a);
    if (e != cudaSuccess) return e;
    return launch_join<F16, D>(a, int(ctas), 8 * NT, s);
}

// Query rows of a key head up to which the tiles of 8 or 16 are faster than those of 128, whose time does not depend on
// how many are filled.  Measured on 64 contexts of 8K: 16 rows 235 us here and 356 us there, 20 rows (two tiles here) 449
// and 359 us, 48 rows 663 and 364 us.  A tile of 8 rather than 16 for 8 rows and fewer: 4 rows, 64 contexts of 8K to 32K
// tokens, 353 and 537 us.  The contexts' lengths are on the device, so the choice goes by the rows alone.
constexpr int kTensorRows = 16;

template <bool F16, int D>
static cudaError_t launch_attn_rows(const AttnArgs &a, int sms, cudaStream_t s) {
    if (a.T * a.group > kTensorRows) return launch_attn_tc(a, F16, D, sms, s);
    return a.T * a.group <= 8 ? launch_attn<F16, D, 1>(a, sms, s) : launch_attn<F16, D, 2>(a, sms, s);
}

}  // namespace switchsd

using namespace switchsd;

extern "C" size_t switchsd_kv4_attention_workspace_bytes(const switchsd_kv4_attention_params *p) {
    return p && kv4_dim_ok(p->D) ? attn_workspace(p->D, 2) : 0;
}

extern "C" int switchsd_kv4_attention(const switchsd_kv4_attention_params *p) {
    if (!p || !p->q || !p->cache || !p->block_table || !p->lens || !p->new_lens || !p->out || !p->workspace) return SWITCHSD_ERR_ARG;
    if (p->dtype != SWITCHSD_BF16 && p->dtype != SWITCHSD_F16) return SWITCHSD_ERR_ARG;
    if (!aligned16(p->q) || !aligned16(p->cache) || !aligned16(p->out) || !aligned16(p->workspace)) return SWITCHSD_ERR_ARG;
    const int32_t sizes[3] = {p->B, p->T, p->Hq};
    for (int i = 0; i < 3; ++i)
        if (!stride_ok(p->q_stride[i], sizes[i])) return SWITCHSD_ERR_ARG;
    if (p->B < 1 || p->T < 1 || p->Hq < 1 || p->Hkv < 1 || p->Hq % p->Hkv != 0 || p->Hq / p->Hkv > 64 || p->blocks < 1 || p->pages < 1 ||
        !kv4_page_ok(p->page) || !kv4_dim_ok(p->D))
        return SWITCHSD_ERR_SHAPE;
    if (int64_t(p->pages) * p->page > 0x7fffffff || int64_t(p->blocks) * p->page > 0x7fffffff - 1024 || int64_t(p->B) * p->T > 0x7fffffff ||
        int64_t(p->T) * (p->Hq / p->Hkv) > 0x7fffffff)
        return SWITCHSD_ERR_SHAPE;
    if (p->workspace_bytes < switchsd_kv4_attention_workspace_bytes(p)) return SWITCHSD_ERR_ARG;
    AttnArgs a;
    a.q = static_cast<const uint16_t *>(p->q);
    for (int i = 0; i < 3; ++i) a.qs[i] = stride_of(p->q_stride[i], sizes[i]);
    a.cache = static_cast<const uint8_t *>(p->cache);
    a.table = p->block_table;
    a.lens = p->lens;
    a.new_lens = p->new_lens;
    a.out = static_cast<uint16_t *>(p->out);
    a.status = p->status;
    a.desc = static_cast<int4 *>(p->workspace);
    a.part = reinterpret_cast<float *>(a.desc + 2 * kAttnMaxCtas);
    a.B = p->B;
    a.T = p->T;
    a.Hq = p->Hq;
    a.Hkv = p->Hkv;
    a.pages = p->pages;
    a.blocks = p->blocks;
    a.page_shift = log2_of(p->page);
    a.lens_add = p->lens_add;
    a.new_add = p->new_add;
    a.group = p->Hq / p->Hkv;
    a.dim = p->D;
    a.scale = p->scale;
    a.give_up = 0;
    const int sms = sm_count();
    if (sms == 0) return SWITCHSD_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(p->stream);
    cudaError_t e;
    if (p->dtype == SWITCHSD_F16)
        e = p->D == 128 ? launch_attn_rows<true, 128>(a, sms, s) : launch_attn_rows<true, 64>(a, sms, s);
    else
        e = p->D == 128 ? launch_attn_rows<false, 128>(a, sms, s) : launch_attn_rows<false, 64>(a, sms, s);
    return e == cudaSuccess ? SWITCHSD_OK : SWITCHSD_ERR_CUDA;
}
