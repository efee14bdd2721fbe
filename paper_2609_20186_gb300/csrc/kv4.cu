// kv4.cu -- switchsd_kv4_append and switchsd_kv4_read: tokens into and out of the 4-bit paged cache.
//
// A warp takes the keys, another the values, of one head's tokens in one block of eight cache positions (a value word
// holds eight tokens, so one warp writes each word).  For the keys lane 4 t + c holds token t's dimensions 16 c ..
// 16 c + 15 of every group, which are the 2 G words it stores; a group's extreme goes over the quad.  For the values lane
// i holds D / 32 neighbouring dimensions of all eight tokens, which are its words; the eight tokens' extremes go over 16 or
// 32 lanes by halves -- a lane hands on the half of the tokens that it does not keep --, so that each lane ends with one
// token's and works out one scale.
//
// A scale goes by one number a group, max(8 pos, 7 neg) / 56 = max(pos / 7, neg / 8), where the products are exact; the
// maximum and minimum are taken of packed pairs, as they come.
//
// A code is x / s rounded half to even, from x times the reciprocal.  x has at most 11 significant bits and s 7, so a
// quotient that is not half-way between two codes is 2^-12 or more off: rounded to a multiple of 2^-15 first, which takes
// the reciprocal's error away, it stays on its side, and one that is half-way comes out as it is.  Both roundings are
// additions, of 1.5 * 2^8 in the product's instruction and of 1.5 * 2^23 in one more, which leaves the code in the low
// bits; eight of those words times powers of 16 add up to a cache word and a known constant.
//
// What bounds it: instructions (about 20 a value, the read 16; 65 and 60 % of the issue slots) more than memory, 2 bytes
// read and 0.53 written a value (and the other way round for the read).  16 rows of 2048 tokens, 8 heads of 128 dimensions:
// append and read take 74 us, where the bytes alone would take 50; of 1 to 2048 tokens each 56 us (35).  A divided quotient and its comparisons
// took 94 us for the latter, limits on every code, not only those of wide groups, and words read token by token 60 us.
#include <cuda_bf16.h>

#include "kv4.cuh"

namespace switchsd {

constexpr int kUnitThreads = 128;

struct AppendArgs {
    const uint8_t *k, *v;
    int64_t ks[3], vs[3];  // strides in elements: row, token, head
    const int32_t *slots;
    uint8_t *cache;
    uint32_t units;        // B * units_per_row * Hkv, below 2^30
    int32_t T, Hkv, units_per_row, page_shift, total;  // total: pages * page slots
};

struct ReadArgs {
    const uint8_t *cache;
    const int32_t *slots;
    uint8_t *k, *v;        // f16 [B][T][Hkv][D]
    uint32_t units;
    int32_t T, Hkv, units_per_row, page_shift, total;
};

// The unit of a warp: eight tokens from t0 on (some before the row's first or after its last), one head.
struct Unit {
    int64_t b;
    int32_t h, t0;
};
template <class Args>
__device__ __forceinline__ Unit unit_of(const Args &a, uint32_t unit) {
    Unit u;
    const uint32_t rest = unit / uint32_t(a.Hkv);
    u.h = int32_t(unit - rest * uint32_t(a.Hkv));
    u.b = rest / uint32_t(a.units_per_row);
    // Blocks begin where the first token's does: unit i has tokens [8 i - a0, 8 i - a0 + 8), a0 its place in the block.
    u.t0 = 8 * int32_t(rest - uint32_t(u.b) * uint32_t(a.units_per_row)) - (__ldcg(a.slots + u.b * a.T) & 7);
    return u;
}
// The slot of token t, -1 where there is none.
template <class Args>
__device__ __forceinline__ int32_t slot_of(const Args &a, int64_t b, int32_t t) {
    const int32_t slot = t >= 0 && t < a.T ? __ldcg(a.slots + b * a.T + t) : -1;
    return slot < a.total ? slot : -1;
}

// Two 16-bit values of the caller's type, widened.
template <bool F16>
__device__ __forceinline__ float2 widen(uint32_t w) {
    if (F16) return __half22float2(*reinterpret_cast<const __half2 *>(&w));
    return make_float2(bf16_lo(w), bf16_hi(w));
}

// The larger and the smaller of two pairs; a NaN stays.
template <bool F16>
__device__ __forceinline__ uint32_t max_pair(uint32_t a, uint32_t b) {
    uint32_t r;
    if (F16)
        asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <bool F16>
__device__ __forceinline__ uint32_t min_pair(uint32_t a, uint32_t b) {
    uint32_t r;
    if (F16)
        asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else
        asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// max(8 pos, 7 neg) of values whose pairs' maximum and minimum are hi and lo.
template <bool F16>
__device__ __forceinline__ float extreme_of(uint32_t hi, uint32_t lo) {
    const float2 h = widen<F16>(hi), l = widen<F16>(lo);
    return max_nan(max_nan(8.f * max_nan(h.x, h.y), 7.f * max_nan(-l.x, -l.y)), 0.f);
}

// The group's stored scale from its extreme (>= 0 or NaN): rounded up to 7 significant bits.  The division is exact where
// the quotient has 7 bits, so that the rounding never lifts such a scale.
__device__ __forceinline__ __half group_scale(float m) {
    if (m != m) return __ushort_as_half(0x7e00);
    const float s = fminf(__fdiv_rn(m, 56.f), kScaleMax);
    return __float2half_rn(__uint_as_float((__float_as_uint(s) + 0x1ffffu) & ~0x1ffffu));
}

// A group's scale and its reciprocal for the codes: zeros, and so codes of 8, where it is 0 or NaN.  Only in a group whose
// scale was cut off at the largest, lost bits among f16's smallest, or is NaN can a quotient lie outside [-8, 7]: `wide`.
struct Scale {
    float s, r;
    bool wide;
    __device__ explicit Scale(__half h) : s(__half2float(h)), r(0.f) {
        wide = !(s < kScaleMax && (s >= 0x1p-17f || s == 0.f));
        if (s > 0.f)
            r = __frcp_rn(s);
        else
            s = 0.f;
    }
    // x inside what the codes reach, for a wide group
    __device__ static float within(float x, float s) { return fminf(fmaxf(x, -8.f * s), 7.f * s); }
};

// A word of codes from the scaled values, an element at a time: nibble_of(j) is element j's.
__device__ __forceinline__ constexpr int nibble_of(int j) { return (j >> 1) + 4 * (j & 1); }
constexpr uint32_t kCodeBits = 0x4b400000u;  // 1.5 * 2^23: the bits of 1.5 * 2^23 + c are kCodeBits + c
// x's code, its bits on top of kCodeBits
__device__ __forceinline__ uint32_t code_of(float x, float r) { return __float_as_uint(fmaf(x, r, 384.f) + (12582912.f + 8.f - 384.f)); }
__device__ __forceinline__ uint32_t put_code(uint32_t w, uint32_t c, int j) { return w + c * (1u << (4 * nibble_of(j))); }
constexpr uint32_t kNoBits = 0u - kCodeBits * 0x11111111u;  // a word of eight codes begins with it

template <bool F16, int D>
__global__ void __launch_bounds__(kUnitThreads) kv4_append_kernel(const AppendArgs a) {
    using L = Kv4<D>;
    constexpr int G = L::G;
    const int lane = threadIdx.x & 31;
    const uint32_t job = blockIdx.x * (kUnitThreads / kWarp) + (threadIdx.x >> 5);
    pdl_wait();
    pdl_trigger();
    if (job >= 2 * a.units) return;
    const Unit u = unit_of(a, job >> 1);
    const int page = 1 << a.page_shift;
    const size_t head_bytes = size_t(kv4_page_bytes(page, D));
    auto head_of = [&](int32_t slot) { return a.cache + (size_t(slot >> a.page_shift) * a.Hkv + u.h) * head_bytes; };
    if ((job & 1) == 0) {
        // --- keys ---------------------------------------------------------------------------------------------
        const int tq = lane >> 2, c = lane & 3;
        const int32_t t = u.t0 + tq, slot = slot_of(a, u.b, t);
        if (__ballot_sync(kFull, slot >= 0) == 0) return;
        const uint8_t *src = a.k + 2 * (u.b * a.ks[0] + int64_t(t) * a.ks[1] + int64_t(u.h) * a.ks[2]);
        uint4 raw[G][2];
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                raw[g][i] = make_uint4(0, 0, 0, 0);
                if (slot >= 0) raw[g][i] = *reinterpret_cast<const uint4 *>(src + 2 * (64 * g + 16 * c + 8 * i));
            }
        uint32_t words[2 * G];
        __half scales[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const uint32_t v[8] = {raw[g][0].x, raw[g][0].y, raw[g][0].z, raw[g][0].w, raw[g][1].x, raw[g][1].y, raw[g][1].z, raw[g][1].w};
            uint32_t hi = v[0], lo = v[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) {
                hi = max_pair<F16>(hi, v[e]);
                lo = min_pair<F16>(lo, v[e]);
            }
            float m = extreme_of<F16>(hi, lo);
            m = max_nan(m, __shfl_xor_sync(kFull, m, 1));
            m = max_nan(m, __shfl_xor_sync(kFull, m, 2));
            scales[g] = group_scale(m);
            const Scale k(scales[g]);
            auto code = [&](auto value) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t w = kNoBits;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 f = widen<F16>(v[4 * i + e]);
                        w = put_code(put_code(w, code_of(value(f.x), k.r), 2 * e), code_of(value(f.y), k.r), 2 * e + 1);
                    }
                    words[2 * g + i] = w;
                }
            };
            if (__any_sync(kFull, k.wide))
                code([&](float x) { return Scale::within(x, k.s); });
            else
                code([](float x) { return x; });
        }
        if (slot < 0) return;
        uint8_t *head = head_of(slot);
        const int in_page = slot & (page - 1);
        uint8_t *dst = head + size_t(in_page) * L::kRow + c * (8 * G);
        if (G == 2)
            *reinterpret_cast<uint4 *>(dst) = make_uint4(words[0], words[1], words[2 * G - 2], words[2 * G - 1]);
        else
            *reinterpret_cast<uint2 *>(dst) = make_uint2(words[0], words[1]);
        if (c == 0) {
            __half *sc = reinterpret_cast<__half *>(head + L::scales(page) + size_t(in_page) * L::kScales);
#pragma unroll
            for (int g = 0; g < G; ++g) sc[g] = scales[g];
        }
        return;
    }
    // --- values -----------------------------------------------------------------------------------------------
    constexpr int N = D / 32;       // dimensions of a lane
    constexpr int kLanes = 64 / N;  // lanes of a group
    const int32_t slot = slot_of(a, u.b, u.t0 + (lane & 7));  // lane e (mod 8): token t0 + e
    // The block: the slot of its first token.  Tokens that do not stand in their place of it (slots that no map wrote) are
    // left out: their words are another warp's.
    const int32_t begin = slot >= (lane & 7) && ((slot - (lane & 7)) & 7) == 0 ? slot - (lane & 7) : -1;
    const uint32_t can = __ballot_sync(kFull, begin >= 0) & 255u;
    if (can == 0) return;
    const int32_t base = __shfl_sync(kFull, begin, __ffs(int(can)) - 1);
    const uint32_t in = __ballot_sync(kFull, slot >= 0 && slot == base + (lane & 7)) & 255u;  // bit e: token t0 + e
    const uint8_t *src = a.v + 2 * (u.b * a.vs[0] + int64_t(u.t0) * a.vs[1] + int64_t(u.h) * a.vs[2]) + 2 * N * lane;
    uint2 raw[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        raw[e] = make_uint2(0, 0);
        if ((in >> e) & 1) {
            const uint8_t *p = src + 2 * int64_t(e) * a.vs[1];
            if (N == 4)
                raw[e] = *reinterpret_cast<const uint2 *>(p);
            else
                raw[e].x = *reinterpret_cast<const uint32_t *>(p);
        }
    }
    float m[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        m[e] = N == 4 ? extreme_of<F16>(max_pair<F16>(raw[e].x, raw[e].y), min_pair<F16>(raw[e].x, raw[e].y))
                      : extreme_of<F16>(raw[e].x, raw[e].x);
    }
    // by halves: after the three exchanges a lane has the token of its three highest bits in the group
#pragma unroll
    for (int half = 4, bit = kLanes / 2; half > 0; half >>= 1, bit >>= 1) {
        const bool upper = (lane & bit) != 0;
#pragma unroll
        for (int e = 0; e < half; ++e) {
            const float keep = upper ? m[e + half] : m[e], give = upper ? m[e] : m[e + half];
            m[e] = max_nan(keep, __shfl_xor_sync(kFull, give, bit));
        }
    }
#pragma unroll
    for (int bit = kLanes / 16; bit > 0; bit >>= 1) m[0] = max_nan(m[0], __shfl_xor_sync(kFull, m[0], bit));
    const __half mine = group_scale(m[0]);
    const int token = (lane / (kLanes / 8)) & 7;  // whose scale this lane has
    if (lane % (kLanes / 8) == 0 && ((in >> token) & 1)) {
        const int32_t at = base + token;
        reinterpret_cast<__half *>(head_of(at) + L::scales(page) + size_t(at & (page - 1)) * L::kScales)[G + lane / kLanes] = mine;
    }
    const Scale own(mine);
    // Tokens that are not in have no bits here: what is there stays.
    uint32_t words[N], keep = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) words[i] = kNoBits;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (!((in >> e) & 1)) keep |= 0xfu << (4 * nibble_of(e));
    auto code = [&](auto value) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int from = (lane & ~(kLanes - 1)) | (e * (kLanes / 8));
            const float s = __shfl_sync(kFull, own.s, from), r = __shfl_sync(kFull, own.r, from);
            const float2 f = widen<F16>(raw[e].x), f2 = widen<F16>(raw[e].y);
            const float x[4] = {f.x, f.y, f2.x, f2.y};
#pragma unroll
            for (int i = 0; i < N; ++i) words[i] = put_code(words[i], code_of(value(x[i], s), r), e);
        }
    };
    if (__any_sync(kFull, own.wide))
        code([](float x, float s) { return Scale::within(x, s); });
    else
        code([](float x, float) { return x; });
#pragma unroll
    for (int i = 0; i < N; ++i) words[i] &= ~keep;
    uint8_t *dst = head_of(base) + L::values(page) + size_t((base & (page - 1)) >> 3) * L::kBlock + 4 * N * lane;
    if (N == 4) {
        uint4 w = make_uint4(words[0], words[1], words[N - 2], words[N - 1]);
        if (keep) {  // tokens of earlier calls in the same words
            const uint4 old = *reinterpret_cast<const uint4 *>(dst);
            w.x |= old.x & keep;
            w.y |= old.y & keep;
            w.z |= old.z & keep;
            w.w |= old.w & keep;
        }
        *reinterpret_cast<uint4 *>(dst) = w;
    } else {
        uint2 w = make_uint2(words[0], words[1]);
        if (keep) {
            const uint2 old = *reinterpret_cast<const uint2 *>(dst);
            w.x |= old.x & keep;
            w.y |= old.y & keep;
        }
        *reinterpret_cast<uint2 *>(dst) = w;
    }
}

// (c - 8) * scale of a pair of codes in bits 0 .. 3 and 16 .. 19, as f16 numbers: exact.
__device__ __forceinline__ uint32_t pair_value(uint32_t w, __half2 s) {
    const uint32_t magic = (w & 0x000f000fu) | 0x64006400u;  // 1024 + c
    const __half2 c = __hsub2(*reinterpret_cast<const __half2 *>(&magic), __float2half2_rn(1032.f));
    const __half2 v = __hmul2(c, s);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// The same units as the append's; tokens without a slot get zeros.
template <int D>
__global__ void __launch_bounds__(kUnitThreads) kv4_read_kernel(const ReadArgs a) {
    using L = Kv4<D>;
    constexpr int G = L::G;
    const int lane = threadIdx.x & 31;
    const uint32_t job = blockIdx.x * (kUnitThreads / kWarp) + (threadIdx.x >> 5);
    pdl_wait();
    pdl_trigger();
    if (job >= 2 * a.units) return;
    const Unit u = unit_of(a, job >> 1);
    const int page = 1 << a.page_shift;
    const size_t head_bytes = size_t(kv4_page_bytes(page, D));
    auto head_of = [&](int32_t slot) { return a.cache + (size_t(slot >> a.page_shift) * a.Hkv + u.h) * head_bytes; };
    auto out_of = [&](uint8_t *out, int32_t t) { return out + ((size_t(u.b) * a.T + t) * a.Hkv + u.h) * (2 * D); };
    if ((job & 1) == 0) {
        const int c = lane & 3;
        const int32_t t = u.t0 + (lane >> 2), slot = slot_of(a, u.b, t);
        if (t < 0 || t >= a.T) return;
        uint32_t words[2 * G];
        __half2 s[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            words[2 * g] = words[2 * g + 1] = 0x88888888u;  // zeros
            s[g] = __float2half2_rn(0.f);
        }
        if (slot >= 0) {
            const uint8_t *head = head_of(slot);
            const int in_page = slot & (page - 1);
            const uint32_t *w = reinterpret_cast<const uint32_t *>(head + size_t(in_page) * L::kRow + c * (8 * G));
            const __half *sc = reinterpret_cast<const __half *>(head + L::scales(page) + size_t(in_page) * L::kScales);
#pragma unroll
            for (int i = 0; i < 2 * G; ++i) words[i] = w[i];
#pragma unroll
            for (int g = 0; g < G; ++g) s[g] = __half2half2(sc[g]);
        }
        uint8_t *out = out_of(a.k, t);
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t w = words[2 * g + i];
                *reinterpret_cast<uint4 *>(out + 2 * (64 * g + 16 * c + 8 * i)) =
                    make_uint4(pair_value(w, s[g]), pair_value(w >> 4, s[g]), pair_value(w >> 8, s[g]), pair_value(w >> 12, s[g]));
            }
        return;
    }
    constexpr int N = D / 32;  // dimensions of a lane
    const int32_t slot = slot_of(a, u.b, u.t0 + (lane & 7));  // lane e (mod 8): token t0 + e
    const int first = max(0, -u.t0), last = min(8, a.T - u.t0);  // the unit's tokens that there are
    if (first >= last) return;
    const uint32_t filled = __ballot_sync(kFull, slot >= 0) & 255u;
    const int32_t begin = __shfl_sync(kFull, slot - (lane & 7), filled ? __ffs(int(filled)) - 1 : 0);
    const bool block = filled && begin >= 0 && (begin & 7) == 0 && __all_sync(kFull, slot < 0 || slot == begin + (lane & 7));
    uint8_t *out = out_of(a.v, u.t0) + 2 * N * lane;
    const size_t token = size_t(a.Hkv) * (2 * D);
    auto store = [&](int e, const uint32_t (&v)[N / 2]) {
        if (N == 4)
            *reinterpret_cast<uint2 *>(out + int64_t(e) * token) = make_uint2(v[0], v[N / 2 - 1]);
        else
            *reinterpret_cast<uint32_t *>(out + int64_t(e) * token) = v[0];
    };
    if (block) {
        // all in their places of one block: its words and scales are read once
        const uint8_t *head = head_of(begin);
        const int in_page = begin & (page - 1);
        const uint32_t *src = reinterpret_cast<const uint32_t *>(head + L::values(page) + size_t(in_page >> 3) * L::kBlock) + N * lane;
        const __half *sc = reinterpret_cast<const __half *>(head + L::scales(page) + size_t(in_page) * L::kScales) + G + N * lane / 64;
        uint32_t w[N];
        __half s[8];
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = src[i];
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = sc[2 * G * e];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e < first || e >= last) continue;
            const __half2 s2 = __half2half2(s[e]);
            uint32_t v[N / 2];
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const int sh = 4 * nibble_of(e);
                v[i] = (filled >> e) & 1 ? pair_value(((w[2 * i] >> sh) & 15u) | (((w[2 * i + 1] >> sh) & 15u) << 16), s2) : 0u;
            }
            store(e, v);
        }
        return;
    }
#pragma unroll 1
    for (int e = first; e < last; ++e) {
        const int32_t se = __shfl_sync(kFull, slot, e);
        uint32_t v[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) v[i] = 0;
        if (se >= 0) {
            const uint8_t *head = head_of(se);
            const int in_page = se & (page - 1), sh = 4 * nibble_of(in_page & 7);
            const uint32_t *w = reinterpret_cast<const uint32_t *>(head + L::values(page) + size_t(in_page >> 3) * L::kBlock) + N * lane;
            const __half *sc = reinterpret_cast<const __half *>(head + L::scales(page) + size_t(in_page) * L::kScales);
            const __half2 s = __half2half2(sc[G + N * lane / 64]);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) v[i] = pair_value(((w[2 * i] >> sh) & 15u) | (((w[2 * i + 1] >> sh) & 15u) << 16), s);
        }
        store(e, v);
    }
}

}  // namespace switchsd

using namespace switchsd;

extern "C" size_t switchsd_kv4_bytes(int32_t page, int32_t D) {
    return kv4_page_ok(page) && kv4_dim_ok(D) ? size_t(kv4_page_bytes(page, D)) : 0;
}

extern "C" int switchsd_kv4_append(const switchsd_kv4_append_params *p) {
    if (!p || !p->k || !p->v || !p->slots || !p->cache) return SWITCHSD_ERR_ARG;
    if (p->dtype != SWITCHSD_BF16 && p->dtype != SWITCHSD_F16) return SWITCHSD_ERR_ARG;
    if (!aligned16(p->k) || !aligned16(p->v) || !aligned16(p->cache)) return SWITCHSD_ERR_ARG;
    const int32_t sizes[3] = {p->B, p->T, p->Hkv};
    for (int i = 0; i < 3; ++i)
        if (!stride_ok(p->k_stride[i], sizes[i]) || !stride_ok(p->v_stride[i], sizes[i])) return SWITCHSD_ERR_ARG;
    if (p->B < 1 || p->T < 1 || p->Hkv < 1 || p->pages < 1 || !kv4_page_ok(p->page) || !kv4_dim_ok(p->D)) return SWITCHSD_ERR_SHAPE;
    if (int64_t(p->pages) * p->page > 0x7fffffff || int64_t(p->B) * p->T > 0x7fffffff) return SWITCHSD_ERR_SHAPE;
    AppendArgs a;
    a.k = static_cast<const uint8_t *>(p->k);
    a.v = static_cast<const uint8_t *>(p->v);
    for (int i = 0; i < 3; ++i) {
        a.ks[i] = stride_of(p->k_stride[i], sizes[i]);
        a.vs[i] = stride_of(p->v_stride[i], sizes[i]);
    }
    a.slots = p->slots;
    a.cache = static_cast<uint8_t *>(p->cache);
    a.T = p->T;
    a.Hkv = p->Hkv;
    a.units_per_row = int32_t((int64_t(p->T) + 6) / 8 + 1);  // the first block may hold one of the row's tokens only
    const int64_t units = int64_t(p->B) * a.units_per_row;
    if (units >= (int64_t(1) << 30) || units * p->Hkv >= (int64_t(1) << 30)) return SWITCHSD_ERR_SHAPE;
    a.units = uint32_t(units) * uint32_t(p->Hkv);
    a.page_shift = log2_of(p->page);
    a.total = p->pages * p->page;
    const uint32_t ctas = (2 * a.units + kUnitThreads / kWarp - 1) / (kUnitThreads / kWarp);
    cudaStream_t s = static_cast<cudaStream_t>(p->stream);
    const dim3 grid{ctas}, block{unsigned(kUnitThreads)};
    cudaError_t e;
    if (p->dtype == SWITCHSD_F16)
        e = p->D == 128 ? launch_pdl(kv4_append_kernel<true, 128>, grid, block, 0, s, 0u, a)
                        : launch_pdl(kv4_append_kernel<true, 64>, grid, block, 0, s, 0u, a);
    else
        e = p->D == 128 ? launch_pdl(kv4_append_kernel<false, 128>, grid, block, 0, s, 0u, a)
                        : launch_pdl(kv4_append_kernel<false, 64>, grid, block, 0, s, 0u, a);
    return e == cudaSuccess ? SWITCHSD_OK : SWITCHSD_ERR_CUDA;
}

extern "C" int switchsd_kv4_read(const switchsd_kv4_read_params *p) {
    if (!p || !p->cache || !p->slots || !p->out_k || !p->out_v) return SWITCHSD_ERR_ARG;
    if (!aligned16(p->cache) || !aligned16(p->out_k) || !aligned16(p->out_v)) return SWITCHSD_ERR_ARG;
    if (p->B < 1 || p->T < 1 || p->Hkv < 1 || p->pages < 1 || !kv4_page_ok(p->page) || !kv4_dim_ok(p->D)) return SWITCHSD_ERR_SHAPE;
    if (int64_t(p->pages) * p->page > 0x7fffffff || int64_t(p->B) * p->T > 0x7fffffff) return SWITCHSD_ERR_SHAPE;
    ReadArgs a;
    a.cache = static_cast<const uint8_t *>(p->cache);
    a.slots = p->slots;
    a.k = static_cast<uint8_t *>(p->out_k);
    a.v = static_cast<uint8_t *>(p->out_v);
    a.T = p->T;
    a.Hkv = p->Hkv;
    a.units_per_row = int32_t((int64_t(p->T) + 6) / 8 + 1);
    const int64_t units = int64_t(p->B) * a.units_per_row;
    if (units >= (int64_t(1) << 30) || units * p->Hkv >= (int64_t(1) << 30)) return SWITCHSD_ERR_SHAPE;
    a.units = uint32_t(units) * uint32_t(p->Hkv);
    a.page_shift = log2_of(p->page);
    a.total = p->pages * p->page;
    const uint32_t ctas = (2 * a.units + kUnitThreads / kWarp - 1) / (kUnitThreads / kWarp);
    cudaStream_t s = static_cast<cudaStream_t>(p->stream);
    const dim3 grid{ctas}, block{unsigned(kUnitThreads)};
    const cudaError_t e = p->D == 128 ? launch_pdl(kv4_read_kernel<128>, grid, block, 0, s, 0u, a) : launch_pdl(kv4_read_kernel<64>, grid, block, 0, s, 0u, a);
    return e == cudaSuccess ? SWITCHSD_OK : SWITCHSD_ERR_CUDA;
}
