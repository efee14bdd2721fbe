// kv16.cu -- switchsd_kv16_append and switchsd_kv16_read: tokens into and out of the 16-bit paged cache.
//
// Copies.  A cache row is a head's D elements of one token, key or value: 16 or 8 vectors of 16 bytes, one a thread, in the
// cache's page [2][Hkv][page][D].  Rows are counted token by token, keys before values, head by head, so that a warp reads
// what is contiguous in a fused projection; a thread has kFlight rows on their way at once, and a CTA no loop.
//
// Bound: the memory's copy rate.  16 rows of 1 to 2048 tokens, 8 heads x 128, append and read: 58 us for 332 MB (84 % of the
// rate of a plain copy); the rest is the CTAs of tokens that are not there (half of them) and two launches.  64 rows of 1 to
// 17 tokens: 5.6 us, two launches' latency.  kFlight 1 / 2 / 8: 84 / 62 / 66 us and 4.5 / 5.8 / 7.4.  A thread that keeps its
// place in the token and goes from token to token, with half of the address arithmetic: 59.5, so it is not that.
#include "kv4.cuh"

namespace switchsd {

constexpr int kCopyThreads = 256;
constexpr int kFlight = 4;  // rows of a thread

// n / d for n < 2^31 by a multiplication: m = ceil(2^(31 + s) / d) with 2^s >= d > 2^(s - 1), whose error times n stays below 1.
struct Divisor {
    uint64_t m;
    uint32_t d, shift;
    Divisor() = default;
    explicit Divisor(uint32_t n) : d(n), shift(31) {
        while ((uint64_t(1) << (shift - 31)) < n) ++shift;
        m = ((uint64_t(1) << shift) + n - 1) / n;
    }
    __device__ uint32_t of(uint32_t n) const { return uint32_t((uint64_t(n) * m) >> shift); }
};

struct CopyArgs {
    uint8_t *k, *v;        // [B][T][Hkv][D]
    int64_t ks[3], vs[3];  // strides in elements
    const int32_t *slots;
    uint8_t *cache;
    uint32_t rows;         // B * T * 2 * Hkv, below 2^31
    Divisor by_heads, by_tokens;
    int32_t Hkv, page_shift, total;
};

template <int D, bool APPEND>
__global__ void __launch_bounds__(kCopyThreads) kv16_copy_kernel(const CopyArgs a) {
    constexpr int V = D / 8, kStep = kCopyThreads / V;  // vectors of a row, rows of a CTA's pass
    const int vec = threadIdx.x % V;
    const uint32_t row0 = blockIdx.x * uint32_t(kFlight * kStep) + threadIdx.x / V;
    uint8_t *outer[kFlight], *inner[kFlight];
    uint4 x[kFlight];
    pdl_wait();
    pdl_trigger();
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
        const uint32_t row = row0 + uint32_t(j * kStep);
        outer[j] = inner[j] = nullptr;
        if (row >= a.rows) continue;
        const uint32_t half_token = a.by_heads.of(row), h = row - half_token * uint32_t(a.Hkv), token = half_token >> 1, half = half_token & 1;
        const uint32_t b = a.by_tokens.of(token), t = token - b * a.by_tokens.d;
        const int64_t *s = half ? a.vs : a.ks;
        outer[j] = (half ? a.v : a.k) + 2 * (b * s[0] + t * s[1] + h * s[2]) + 16 * vec;
        const int32_t slot = __ldcg(a.slots + token);
        if (uint32_t(slot) >= uint32_t(a.total)) continue;
        const size_t page = uint32_t(slot) >> a.page_shift, in = uint32_t(slot) & ((1u << a.page_shift) - 1);
        inner[j] = a.cache + 2 * D * ((((page * 2 + half) * a.Hkv + h) << a.page_shift) + in) + 16 * vec;
    }
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
        x[j] = make_uint4(0, 0, 0, 0);
        if (inner[j]) x[j] = __ldcs(reinterpret_cast<const uint4 *>(APPEND ? outer[j] : inner[j]));
    }
#pragma unroll
    for (int j = 0; j < kFlight; ++j) {
        uint8_t *to = APPEND ? inner[j] : outer[j];
        if (to) *reinterpret_cast<uint4 *>(to) = x[j];
    }
}

template <bool APPEND>
static int copy(CopyArgs &a, int32_t B, int32_t T, int32_t Hkv, int32_t D, int32_t page, int32_t pages, void *stream) {
    a.rows = uint32_t(B) * uint32_t(T) * 2 * uint32_t(Hkv);
    a.by_heads = Divisor(uint32_t(Hkv));
    a.by_tokens = Divisor(uint32_t(T));
    a.Hkv = Hkv;
    a.page_shift = log2_of(page);
    a.total = pages * page;
    const uint32_t per = kFlight * uint32_t(kCopyThreads * 8 / D);
    const dim3 grid{(a.rows + per - 1) / per}, block{unsigned(kCopyThreads)};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = D == 128 ? launch_pdl(kv16_copy_kernel<128, APPEND>, grid, block, 0, s, 0u, a) : launch_pdl(kv16_copy_kernel<64, APPEND>, grid, block, 0, s, 0u, a);
    return e == cudaSuccess ? SWITCHSD_OK : SWITCHSD_ERR_CUDA;
}

static bool copy_shape_ok(int32_t B, int32_t T, int32_t Hkv, int32_t D, int32_t page, int32_t pages) {
    return B >= 1 && T >= 1 && Hkv >= 1 && pages >= 1 && kv4_page_ok(page) && kv4_dim_ok(D) && int64_t(pages) * page <= 0x7fffffff &&
           int64_t(B) * T < (int64_t(1) << 30) && int64_t(B) * T * Hkv < (int64_t(1) << 30);
}

}  // namespace switchsd

using namespace switchsd;

extern "C" int switchsd_kv16_append(const switchsd_kv16_append_params *p) {
    if (!p || !p->k || !p->v || !p->slots || !p->cache) return SWITCHSD_ERR_ARG;
    if (p->dtype != SWITCHSD_BF16 && p->dtype != SWITCHSD_F16) return SWITCHSD_ERR_ARG;
    if (!aligned16(p->k) || !aligned16(p->v) || !aligned16(p->cache)) return SWITCHSD_ERR_ARG;
    const int32_t sizes[3] = {p->B, p->T, p->Hkv};
    for (int i = 0; i < 3; ++i)
        if (!stride_ok(p->k_stride[i], sizes[i]) || !stride_ok(p->v_stride[i], sizes[i])) return SWITCHSD_ERR_ARG;
    if (!copy_shape_ok(p->B, p->T, p->Hkv, p->D, p->page, p->pages)) return SWITCHSD_ERR_SHAPE;
    CopyArgs a;
    a.k = static_cast<uint8_t *>(const_cast<void *>(p->k));
    a.v = static_cast<uint8_t *>(const_cast<void *>(p->v));
    for (int i = 0; i < 3; ++i) {
        a.ks[i] = stride_of(p->k_stride[i], sizes[i]);
        a.vs[i] = stride_of(p->v_stride[i], sizes[i]);
    }
    a.slots = p->slots;
    a.cache = static_cast<uint8_t *>(p->cache);
    return copy<true>(a, p->B, p->T, p->Hkv, p->D, p->page, p->pages, p->stream);
}

extern "C" int switchsd_kv16_read(const switchsd_kv16_read_params *p) {
    if (!p || !p->cache || !p->slots || !p->out_k || !p->out_v) return SWITCHSD_ERR_ARG;
    if (!aligned16(p->cache) || !aligned16(p->out_k) || !aligned16(p->out_v)) return SWITCHSD_ERR_ARG;
    if (!copy_shape_ok(p->B, p->T, p->Hkv, p->D, p->page, p->pages)) return SWITCHSD_ERR_SHAPE;
    CopyArgs a;
    a.k = static_cast<uint8_t *>(p->out_k);
    a.v = static_cast<uint8_t *>(p->out_v);
    const int64_t dense[3] = {int64_t(p->T) * p->Hkv * p->D, int64_t(p->Hkv) * p->D, p->D};
    for (int i = 0; i < 3; ++i) a.ks[i] = a.vs[i] = dense[i];
    a.slots = p->slots;
    a.cache = static_cast<uint8_t *>(const_cast<void *>(p->cache));
    return copy<false>(a, p->B, p->T, p->Hkv, p->D, p->page, p->pages, p->stream);
}
