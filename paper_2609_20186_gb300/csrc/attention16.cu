// attention16.cu -- switchsd_kv16_attention: attention of a step's new tokens over the 16-bit paged cache.
//
// The plain form: a warp a (token, query head), lane i holding D / 32 dimensions, one pass over the keys with the running
// maximum and sum.
#include "attention.cuh"

namespace switchsd {

constexpr int kPlainThreads = 128;

template <bool F16, int D>
__global__ void __launch_bounds__(kPlainThreads) attn16_plain_kernel(const AttnArgs a) {
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31;
    pdl_wait();
    pdl_trigger();
    const int64_t warps = int64_t(gridDim.x) * (kPlainThreads / kWarp), first = (int64_t(blockIdx.x) * kPlainThreads + threadIdx.x) / kWarp;
    if (a.status && blockIdx.x == 0)
        for (int b = threadIdx.x; b < a.B; b += kPlainThreads) {
            int32_t len, nw;
            a.status[b] = row_lengths(a, b, len, nw) ? SWITCHSD_ROW_OK : SWITCHSD_ROW_BAD_LEN;
        }
    for (int64_t i = first; i < int64_t(a.B) * a.T * a.Hq; i += warps) {
        const int h = int(i % a.Hq), t = int(i / a.Hq % a.T), b = int(i / a.Hq / a.T), hk = h / a.group;
        int32_t len, nw;
        row_lengths(a, b, len, nw);
        float m = -INFINITY, l = 0.f, o[E], q[E];
        for (int e = 0; e < E; ++e) {
            o[e] = 0.f;
            q[e] = t < nw ? widen1<F16>(a.q[b * a.qs[0] + t * a.qs[1] + h * a.qs[2] + lane * E + e]) : 0.f;
        }
        const int32_t end = t < nw ? len + t + 1 : 0, mask = (1 << a.page_shift) - 1;
        for (int32_t j = 0; j < end; ++j) {
            const int32_t page = __ldcg(a.table + size_t(b) * a.blocks + (j >> a.page_shift));
            if (uint32_t(page) >= uint32_t(a.pages)) continue;
            const uint16_t *k = reinterpret_cast<const uint16_t *>(a.cache) + (((size_t(page) * 2 * a.Hkv + hk) << a.page_shift) + (j & mask)) * D + lane * E;
            const uint16_t *v = k + (size_t(a.Hkv) << a.page_shift) * D;
            float s = 0.f;
            for (int e = 0; e < E; ++e) s = fmaf(q[e], widen1<F16>(k[e]), s);
            s = warp_sum_f32(s) * a.scale;
            if (!(s <= m)) {
                const float f = expf(m - s);
                m = s;
                l *= f;
                for (int e = 0; e < E; ++e) o[e] *= f;
            }
            const float p = expf(s - m);
            l += p;
            for (int e = 0; e < E; ++e) o[e] = fmaf(p, widen1<F16>(v[e]), o[e]);
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        for (int e = 0; e < E; ++e) a.out[i * D + lane * E + e] = narrow1<F16>(o[e] * inv);
    }
}

}  // namespace switchsd

using namespace switchsd;

extern "C" size_t switchsd_kv16_attention_workspace_bytes(const switchsd_kv16_attention_params *p) {
    return p && kv4_dim_ok(p->D) ? 16 : 0;
}

extern "C" int switchsd_kv16_attention(const switchsd_kv16_attention_params *p) {
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
    if (p->workspace_bytes < switchsd_kv16_attention_workspace_bytes(p)) return SWITCHSD_ERR_ARG;
    AttnArgs a = {};
    a.q = static_cast<const uint16_t *>(p->q);
    for (int i = 0; i < 3; ++i) a.qs[i] = stride_of(p->q_stride[i], sizes[i]);
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
    a.group = p->Hq / p->Hkv;
    a.dim = p->D;
    a.scale = p->scale;
    cudaStream_t s = static_cast<cudaStream_t>(p->stream);
    const dim3 grid(unsigned(std::min<int64_t>(int64_t(1) << 20, (int64_t(p->B) * p->T * p->Hq + 3) / 4))), block(kPlainThreads);
    cudaError_t e;
    if (p->dtype == SWITCHSD_F16)
        e = p->D == 128 ? launch_pdl(attn16_plain_kernel<true, 128>, grid, block, 0, s, 0u, a) : launch_pdl(attn16_plain_kernel<true, 64>, grid, block, 0, s, 0u, a);
    else
        e = p->D == 128 ? launch_pdl(attn16_plain_kernel<false, 128>, grid, block, 0, s, 0u, a) : launch_pdl(attn16_plain_kernel<false, 64>, grid, block, 0, s, 0u, a);
    return e == cudaSuccess ? SWITCHSD_OK : SWITCHSD_ERR_CUDA;
}
