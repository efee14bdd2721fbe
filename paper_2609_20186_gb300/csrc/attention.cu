// attention.cu -- switchsd_kv4_attention: attention of a step's new tokens over the 4-bit paged cache.
#include <cuda_bf16.h>

#include <algorithm>

#include "kv4.cuh"

namespace switchsd {

struct AttnArgs {
    const uint16_t *q;
    int64_t qs[3];
    const uint8_t *cache;
    const int32_t *table, *lens, *new_lens;
    uint16_t *out;
    int32_t *status;
    int32_t B, T, Hq, Hkv, pages, blocks, page_shift, lens_add, new_add;
    float scale;
};

// A row's lengths, or false where they are bad.
__device__ __forceinline__ bool row_lengths(const AttnArgs &a, int b, int32_t &len, int32_t &nw) {
    const int64_t l = int64_t(__ldcg(a.lens + b)) + a.lens_add, n = int64_t(__ldcg(a.new_lens + b)) + a.new_add;
    const bool ok = l >= 0 && n >= 0 && n <= a.T && l + n <= (int64_t(a.blocks) << a.page_shift);
    len = ok ? int32_t(l) : 0;
    nw = ok ? int32_t(n) : 0;
    return ok;
}

// One warp per (row, token, query head), over the keys one by one.
template <bool F16, int D>
__global__ void __launch_bounds__(128) attn_simple_kernel(const AttnArgs a) {
    using L = Kv4<D>;
    constexpr int N = D / 32;
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const int64_t w = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 5);
    if (w >= int64_t(a.B) * a.T * a.Hq) return;
    const int h = int(w % a.Hq), t = int(w / a.Hq % a.T), b = int(w / a.Hq / a.T);
    int32_t len, nw;
    const bool ok = row_lengths(a, b, len, nw);
    if (a.status && h == 0 && t == 0 && lane == 0) a.status[b] = ok ? SWITCHSD_ROW_OK : SWITCHSD_ROW_BAD_LEN;
    const int page = 1 << a.page_shift, hk = h / (a.Hq / a.Hkv);
    const uint16_t *q = a.q + b * a.qs[0] + t * a.qs[1] + h * a.qs[2] + N * lane;
    float qf[N], o[N], m = -1e30f, l = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        qf[i] = (F16 ? __half2float(__ushort_as_half(q[i])) : bf16_lo(q[i])) * a.scale;
        o[i] = 0.f;
    }
    const int dw = N * lane / 8, g = dw >> 3;
    const int word = ((dw & 7) >> 1) * (2 * L::G) + 2 * g + (dw & 1);
    const int32_t n = t < nw ? len + t + 1 : 0;
    for (int32_t j = 0; j < n; ++j) {
        const int32_t pg = __ldcg(a.table + size_t(b) * a.blocks + (j >> a.page_shift));
        if (uint32_t(pg) >= uint32_t(a.pages)) continue;
        const int in = j & (page - 1);
        const uint8_t *src = a.cache + (size_t(pg) * a.Hkv + hk) * size_t(kv4_page_bytes(page, D));
        const __half *sc = reinterpret_cast<const __half *>(src + L::scales(page) + size_t(in) * L::kScales);
        const uint32_t kw = *reinterpret_cast<const uint32_t *>(src + size_t(in) * L::kRow + 4 * word);
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = (N * lane + i) & 7;
            x += qf[i] * (float((kw >> (4 * ((e >> 1) + 4 * (e & 1)))) & 15u) - 8.f);
        }
        x = warp_sum_f32(x * __half2float(sc[g]));
        const float mn = fmaxf(m, x), f = __expf(m - mn), p = __expf(x - mn);
        m = mn;
        l = l * f + p;
        const uint32_t *vw = reinterpret_cast<const uint32_t *>(src + L::values(page) + size_t(in >> 3) * L::kBlock) + N * lane;
        const int shift = 4 * (((in & 7) >> 1) + 4 * (in & 1));
        const float pv = p * __half2float(sc[L::G + g]);
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = o[i] * f + pv * (float((vw[i] >> shift) & 15u) - 8.f);
    }
    const float inv = l > 0.f ? 1.f / l : (l != l ? l : 0.f);
    uint16_t *out = a.out + ((size_t(b) * a.T + t) * a.Hq + h) * D + N * lane;
#pragma unroll
    for (int i = 0; i < N; ++i)
        out[i] = F16 ? __half_as_ushort(__float2half_rn(o[i] * inv)) : __bfloat16_as_ushort(__float2bfloat16_rn(o[i] * inv));
}

}  // namespace switchsd

using namespace switchsd;

extern "C" size_t switchsd_kv4_attention_workspace_bytes(const switchsd_kv4_attention_params *p) {
    return p ? 16 : 0;
}

extern "C" int switchsd_kv4_attention(const switchsd_kv4_attention_params *p) {
    if (!p || !p->q || !p->cache || !p->block_table || !p->lens || !p->new_lens || !p->out || !p->workspace) return SWITCHSD_ERR_ARG;
    if (p->dtype != SWITCHSD_BF16 && p->dtype != SWITCHSD_F16) return SWITCHSD_ERR_ARG;
    if (!aligned16(p->q) || !aligned16(p->cache) || !aligned16(p->out) || !aligned16(p->workspace)) return SWITCHSD_ERR_ARG;
    for (int i = 0; i < 3; ++i)
        if (p->q_stride[i] % 8 != 0 || p->q_stride[i] < 0) return SWITCHSD_ERR_ARG;
    if (p->B < 1 || p->T < 1 || p->Hq < 1 || p->Hkv < 1 || p->Hq % p->Hkv != 0 || p->Hq / p->Hkv > 64 || p->blocks < 1 || p->pages < 1 ||
        !kv4_page_ok(p->page) || !kv4_dim_ok(p->D))
        return SWITCHSD_ERR_SHAPE;
    if (int64_t(p->pages) * p->page > 0x7fffffff || int64_t(p->blocks) * p->page > 0x7fffffff || int64_t(p->B) * p->T > 0x7fffffff)
        return SWITCHSD_ERR_SHAPE;
    if (p->workspace_bytes < switchsd_kv4_attention_workspace_bytes(p)) return SWITCHSD_ERR_ARG;
    AttnArgs a;
    a.q = static_cast<const uint16_t *>(p->q);
    for (int i = 0; i < 3; ++i) a.qs[i] = p->q_stride[i];
    a.cache = static_cast<const uint8_t *>(p->cache);
    a.table = p->block_table;
    a.lens = p->lens;
    a.new_lens = p->new_lens;
    a.out = static_cast<uint16_t *>(p->out);
    a.status = p->status;
    a.B = p->B;
    a.T = p->T;
    a.Hq = p->Hq;
    a.Hkv = p->Hkv;
    a.pages = p->pages;
    a.blocks = p->blocks;
    a.page_shift = log2_of(p->page);
    a.lens_add = p->lens_add;
    a.new_add = p->new_add;
    a.scale = p->scale;
    const int64_t ctas = (int64_t(p->B) * p->T * p->Hq + 3) / 4;
    if (ctas > 0x7fffffff) return SWITCHSD_ERR_SHAPE;
    cudaStream_t s = static_cast<cudaStream_t>(p->stream);
    const dim3 grid{unsigned(ctas)}, block{128u};
    cudaError_t e;
    if (p->dtype == SWITCHSD_F16)
        e = p->D == 128 ? launch_pdl(attn_simple_kernel<true, 128>, grid, block, 0, s, 0u, a) : launch_pdl(attn_simple_kernel<true, 64>, grid, block, 0, s, 0u, a);
    else
        e = p->D == 128 ? launch_pdl(attn_simple_kernel<false, 128>, grid, block, 0, s, 0u, a) : launch_pdl(attn_simple_kernel<false, 64>, grid, block, 0, s, 0u, a);
    return e == cudaSuccess ? SWITCHSD_OK : SWITCHSD_ERR_CUDA;
}
