// kv4.cu -- switchsd_kv4_append and switchsd_kv4_read: tokens into and out of the 4-bit paged cache.
//
// A warp takes one head's tokens of one block of eight cache positions (a value word holds eight tokens, so one warp
// writes each word).  For the keys lane 4 t + c holds token t's dimensions 16 c .. 16 c + 15 of every group, which are
// the 4 G words it stores; a group's extremes go over the quad.  For the values lane i holds D / 32 neighbouring
// dimensions of all eight tokens, which are its words; a group's extremes go over 16 or 32 lanes.
#include <cuda_bf16.h>

#include "kv4.cuh"

namespace switchsd {

constexpr int kAppendThreads = 128;

struct AppendArgs {
    const uint8_t *k, *v;
    int64_t ks[3], vs[3];  // strides in elements: row, token, head
    const int32_t *slots;
    uint8_t *cache;
    int64_t units;         // B * units_per_row * Hkv
    int32_t T, Hkv, units_per_row, page_shift, total;  // total: pages * page slots
};

// Two 16-bit values of the caller's type, widened.
template <bool F16>
__device__ __forceinline__ float2 widen(uint32_t w) {
    if (F16) {
        return __half22float2(*reinterpret_cast<const __half2 *>(&w));
    }
    return make_float2(bf16_lo(w), bf16_hi(w));
}

// max that keeps a NaN.
__device__ __forceinline__ float max_nan(float a, float b) { return (a > b || a != a) ? a : b; }

// The group's stored scale from its extremes: max(pos / 7, neg / 8) rounded up to 7 significant bits.  pos, neg >= 0
// or NaN.  The divisions are exact where the quotient has 7 bits, so that the rounding never lifts such a scale.
__device__ __forceinline__ __half group_scale(float pos, float neg) {
    float s = max_nan(__fdiv_rn(pos, 7.f), neg * 0.125f);
    if (s != s) return __ushort_as_half(0x7e00);
    s = fminf(s, kScaleMax);
    return __float2half_rn(__uint_as_float((__float_as_uint(s) + 0x1ffffu) & ~0x1ffffu));
}

// The code of x under scale s: round(x / s) to even, in 0 .. 15; 8 where s is 0 or NaN.
__device__ __forceinline__ uint32_t code_of(float x, float s) {
    if (!(s > 0.f)) return 8u;
    const float q = fminf(fmaxf(rintf(__fdiv_rn(x, s)), -8.f), 7.f);
    return uint32_t(int(q) + 8);
}

__device__ __forceinline__ constexpr int nibble_of(int j) { return (j >> 1) + 4 * (j & 1); }

template <bool F16, int D>
__global__ void __launch_bounds__(kAppendThreads) kv4_append_kernel(const AppendArgs a) {
    using L = Kv4<D>;
    constexpr int G = L::G;
    const int lane = threadIdx.x & 31;
    const int64_t unit = int64_t(blockIdx.x) * (kAppendThreads / kWarp) + (threadIdx.x >> 5);
    pdl_wait();
    pdl_trigger();
    if (unit >= a.units) return;
    const int h = int(unit % a.Hkv);
    const int u = int((unit / a.Hkv) % a.units_per_row);
    const int64_t b = unit / a.Hkv / a.units_per_row;
    const int32_t *slots = a.slots + b * a.T;
    // Blocks begin where the first token's does: unit u has tokens [8 u - a0, 8 u - a0 + 8), a0 its place in the block.
    const int32_t a0 = __ldcg(slots) & 7;
    const int32_t t0 = 8 * u - a0;
    const int tq = lane >> 2, c = lane & 3;
    // lane 4 t + c looks at token t0 + t
    const int32_t t = t0 + tq;
    const int32_t slot = t >= 0 && t < a.T ? __ldcg(slots + t) : -1;
    const bool live = slot >= 0 && slot < a.total;
    const uint32_t any = __ballot_sync(kFull, live);
    if (any == 0) return;
    const int page = 1 << a.page_shift;
    const size_t head_bytes = size_t(kv4_page_bytes(page, D));
    // --- keys -------------------------------------------------------------------------------------------------
    uint8_t *mine = a.cache + (size_t(live ? slot >> a.page_shift : 0) * a.Hkv + h) * head_bytes;
    const int in_page = slot & (page - 1);
    {
        uint32_t words[2 * G];
        __half scales[G];
        const uint8_t *src = a.k + 2 * (b * a.ks[0] + int64_t(t) * a.ks[1] + int64_t(h) * a.ks[2]);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float x[16];
            float pos = 0.f, neg = 0.f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint4 r = make_uint4(0, 0, 0, 0);
                if (live) r = *reinterpret_cast<const uint4 *>(src + 2 * (64 * g + 16 * c + 8 * i));
                const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 f = widen<F16>(w[e]);
                    x[8 * i + 2 * e] = f.x;
                    x[8 * i + 2 * e + 1] = f.y;
                }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                pos = max_nan(x[e], pos);
                neg = max_nan(-x[e], neg);
            }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                pos = max_nan(pos, __shfl_xor_sync(kFull, pos, o));
                neg = max_nan(neg, __shfl_xor_sync(kFull, neg, o));
            }
            scales[g] = group_scale(pos, neg);
            const float s = __half2float(scales[g]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t w = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) w |= code_of(x[8 * i + e], s) << (4 * nibble_of(e));
                words[2 * g + i] = w;
            }
        }
        if (live) {
            uint8_t *dst = mine + size_t(in_page) * L::kRow + c * (8 * G);
            if (G == 2)
                *reinterpret_cast<uint4 *>(dst) = make_uint4(words[0], words[1], words[2 * G - 2], words[2 * G - 1]);
            else
                *reinterpret_cast<uint2 *>(dst) = make_uint2(words[0], words[1]);
            if (c == 0) {
                __half *sc = reinterpret_cast<__half *>(mine + L::scales(page) + size_t(in_page) * L::kScales);
#pragma unroll
                for (int g = 0; g < G; ++g) sc[g] = scales[g];
            }
        }
    }
    // --- values -----------------------------------------------------------------------------------------------
    constexpr int N = D / 32;  // dimensions of a lane
    uint32_t words[N], keep = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) words[i] = 0;
    int32_t base = -1;         // the block: slot of its first token
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int32_t se = __shfl_sync(kFull, slot, 4 * e);
        const bool le = se >= 0 && se < a.total;
        // A token that does not stand e places into the first one's block (slots that no map wrote) is left out: its
        // word is another warp's.
        if (le && base < 0 && se >= e && ((se - e) & 7) == 0) base = se - e;
        const bool in = le && se == base + e;
        float x[N];
        float pos = 0.f, neg = 0.f;
        const uint8_t *src = a.v + 2 * (b * a.vs[0] + int64_t(t0 + e) * a.vs[1] + int64_t(h) * a.vs[2]) + 2 * N * lane;
        uint2 r = make_uint2(0, 0);
        if (in) {
            if (N == 4)
                r = *reinterpret_cast<const uint2 *>(src);
            else
                r.x = *reinterpret_cast<const uint32_t *>(src);
        }
        {
            const float2 f = widen<F16>(r.x);
            x[0] = f.x;
            x[1] = f.y;
            if (N == 4) {
                const float2 f2 = widen<F16>(r.y);
                x[N - 2] = f2.x;
                x[N - 1] = f2.y;
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            pos = max_nan(x[i], pos);
            neg = max_nan(-x[i], neg);
        }
#pragma unroll
        for (int o = 1; o < 64 / N; o <<= 1) {
            pos = max_nan(pos, __shfl_xor_sync(kFull, pos, o));
            neg = max_nan(neg, __shfl_xor_sync(kFull, neg, o));
        }
        const __half sh = group_scale(pos, neg);
        const float s = __half2float(sh);
        if (in) {
#pragma unroll
            for (int i = 0; i < N; ++i) words[i] |= code_of(x[i], s) << (4 * nibble_of(e));
            if ((lane & (64 / N - 1)) == 0) {
                uint8_t *at = a.cache + (size_t(se >> a.page_shift) * a.Hkv + h) * head_bytes;
                reinterpret_cast<__half *>(at + L::scales(page) + size_t(se & (page - 1)) * L::kScales)[G + lane / (64 / N)] = sh;
            }
        } else {
            keep |= 0xfu << (4 * nibble_of(e));
        }
    }
    if (base < 0) return;
    uint8_t *dst = a.cache + (size_t(base >> a.page_shift) * a.Hkv + h) * head_bytes + L::values(page) +
                   size_t((base & (page - 1)) >> 3) * L::kBlock + 4 * N * lane;
    if (N == 4) {
        uint4 w = make_uint4(words[0], words[1], words[N - 2], words[N - 1]);
        if (keep) {
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

struct ReadArgs {
    const uint8_t *cache;
    const int32_t *slots;
    uint8_t *k, *v;   // f16 [tokens][Hkv][D]
    int64_t n;        // tokens * Hkv * D / 8
    int32_t Hkv, page_shift, total;
};

// A thread reads eight dimensions of one token's key and value.
template <int D>
__global__ void __launch_bounds__(256) kv4_read_kernel(const ReadArgs a) {
    using L = Kv4<D>;
    pdl_wait();
    pdl_trigger();
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= a.n) return;
    const int dw = int(i % (D / 8));
    const int64_t th = i / (D / 8);
    const int h = int(th % a.Hkv);
    const int32_t slot = __ldcg(a.slots + th / a.Hkv);
    __half ok[8], ov[8];
    if (slot >= 0 && slot < a.total) {
        const int page = 1 << a.page_shift, in = slot & (page - 1), g = dw >> 3;
        const uint8_t *src = a.cache + (size_t(slot >> a.page_shift) * a.Hkv + h) * size_t(kv4_page_bytes(page, D));
        const __half *sc = reinterpret_cast<const __half *>(src + L::scales(page) + size_t(in) * L::kScales);
        const int word = ((dw & 7) >> 1) * (2 * L::G) + 2 * g + (dw & 1);
        const uint32_t w = *reinterpret_cast<const uint32_t *>(src + size_t(in) * L::kRow + 4 * word);
        const uint32_t *vw = reinterpret_cast<const uint32_t *>(src + L::values(page) + size_t(in >> 3) * L::kBlock) + 8 * dw;
        const float ks = __half2float(sc[g]), vs = __half2float(sc[L::G + g]);
        const int shift = 4 * (((in & 7) >> 1) + 4 * (in & 1));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            ok[j] = __float2half_rn((float((w >> (4 * nibble_of(j))) & 15u) - 8.f) * ks);
            ov[j] = __float2half_rn((float((vw[j] >> shift) & 15u) - 8.f) * vs);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) ok[j] = ov[j] = __ushort_as_half(0);
    }
    *reinterpret_cast<uint4 *>(a.k + 16 * i) = *reinterpret_cast<uint4 *>(ok);
    *reinterpret_cast<uint4 *>(a.v + 16 * i) = *reinterpret_cast<uint4 *>(ov);
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
    for (int i = 0; i < 3; ++i)
        if (p->k_stride[i] % 8 != 0 || p->v_stride[i] % 8 != 0 || p->k_stride[i] < 0 || p->v_stride[i] < 0) return SWITCHSD_ERR_ARG;
    if (p->B < 1 || p->T < 1 || p->Hkv < 1 || p->pages < 1 || !kv4_page_ok(p->page) || !kv4_dim_ok(p->D)) return SWITCHSD_ERR_SHAPE;
    if (int64_t(p->pages) * p->page > 0x7fffffff || int64_t(p->B) * p->T > 0x7fffffff) return SWITCHSD_ERR_SHAPE;
    AppendArgs a;
    a.k = static_cast<const uint8_t *>(p->k);
    a.v = static_cast<const uint8_t *>(p->v);
    for (int i = 0; i < 3; ++i) {
        a.ks[i] = p->k_stride[i];
        a.vs[i] = p->v_stride[i];
    }
    a.slots = p->slots;
    a.cache = static_cast<uint8_t *>(p->cache);
    a.T = p->T;
    a.Hkv = p->Hkv;
    a.units_per_row = (p->T - 1 + 7) / 8 + 1;  // the first block may hold one of the row's tokens only
    a.units = int64_t(p->B) * a.units_per_row * p->Hkv;
    a.page_shift = log2_of(p->page);
    a.total = p->pages * p->page;
    const int64_t ctas = (a.units + kAppendThreads / kWarp - 1) / (kAppendThreads / kWarp);
    if (ctas > 0x7fffffff) return SWITCHSD_ERR_SHAPE;
    cudaStream_t s = static_cast<cudaStream_t>(p->stream);
    const dim3 grid{unsigned(ctas)}, block{unsigned(kAppendThreads)};
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
    a.n = int64_t(p->B) * p->T * p->Hkv * (p->D / 8);
    a.Hkv = p->Hkv;
    a.page_shift = log2_of(p->page);
    a.total = p->pages * p->page;
    const int64_t ctas = (a.n + 255) / 256;
    if (ctas > 0x7fffffff) return SWITCHSD_ERR_SHAPE;
    cudaStream_t s = static_cast<cudaStream_t>(p->stream);
    const cudaError_t e = p->D == 128 ? launch_pdl(kv4_read_kernel<128>, dim3(unsigned(ctas)), dim3(256u), 0, s, 0u, a)
                                      : launch_pdl(kv4_read_kernel<64>, dim3(unsigned(ctas)), dim3(256u), 0, s, 0u, a);
    return e == cudaSuccess ? SWITCHSD_OK : SWITCHSD_ERR_CUDA;
}
