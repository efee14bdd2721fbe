// logits.cu -- switchsd_logits: penalties for repeated tokens, biases and grammar masks on the logits of B rows and T
// positions, and every position's greedy token.
//
// A cluster of kLogitParts CTAs takes one row and a range of its positions, each CTA a slice of the vocabulary.  It
// counts the row's context for its slice in shared memory (one word a token: output occurrences, and flags), marks the
// tokens that need more than a comparison in a bit map -- seen, biased or in the draft --, and then streams the slice
// of every position once.  The CTAs' best tokens meet in the first one's shared memory.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "common.cuh"
#include "switchsd_target.h"

namespace switchsd {

constexpr int kLogitParts = 8;
constexpr int kLogitThreads = 512;
constexpr int kLogitWarps = kLogitThreads / kWarp;
constexpr int kLogitRange = 64;             // most positions of a cluster
constexpr uint32_t kSeen = 1u << 31;        // in a token's word: occurs in the context
constexpr uint32_t kInDraft = 1u << 30;     // occurs in the draft
constexpr uint32_t kCount = kInDraft - 1;   // output occurrences in the context

struct LogitArgs {
    const uint8_t *logits;
    uint8_t *out;
    int64_t sb, st, ob, ot;  // strides in elements
    const int32_t *ctx, *lens, *draft, *new_lens, *prompt, *bias_ids;
    const float *rep, *freq, *pres, *bias;
    const uint32_t *mask;
    int32_t *argmax, *status;
    int32_t T, V, cap, draft_stride, new_add, nbias, mask_words;
    int32_t slice;           // tokens of a CTA, a multiple of 64
    int32_t range;           // positions of a cluster
};

template <int DT>
struct Elem;
template <>
struct Elem<SWITCHSD_BF16> {
    using type = uint16_t;
    __device__ static float get(uint16_t v) { return bf16_lo(v); }
    __device__ static uint16_t put(float f) { return __bfloat16_as_ushort(__float2bfloat16_rn(f)); }
};
template <>
struct Elem<SWITCHSD_F16> {
    using type = uint16_t;
    __device__ static float get(uint16_t v) { return __half2float(__ushort_as_half(v)); }
    __device__ static uint16_t put(float f) { return __half_as_ushort(__float2half_rn(f)); }
};
template <>
struct Elem<SWITCHSD_F32> {
    using type = float;
    __device__ static float get(float v) { return v; }
    __device__ static float put(float f) { return f; }
};

// (value, token) as a word whose order is larger value first, then smaller token; 0 is nothing.
__device__ __forceinline__ uint64_t best_key(float v, int32_t id) {
    if (id < 0) return 0;
    const uint32_t u = __float_as_uint(v);
    const uint32_t o = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return (uint64_t(o) << 32) | uint32_t(~uint32_t(id));
}

__device__ __forceinline__ uint64_t warp_max_u64(uint64_t k) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const uint64_t y = __shfl_xor_sync(kFull, k, o);
        k = y > k ? y : k;
    }
    return k;
}

template <int DT>
__global__ void __launch_bounds__(kLogitThreads) logits_kernel(const LogitArgs a) {
    using E = Elem<DT>;
    using elem = typename E::type;
    constexpr int N = 16 / int(sizeof(elem));  // elements of a vector
    extern __shared__ uint32_t smem[];
    __shared__ uint64_t s_best[kLogitRange][kLogitWarps];
    __shared__ uint64_t s_part[kLogitParts][kLogitRange];
    uint32_t *cnt = smem;                                                   // [slice]
    uint32_t *bits = smem + a.slice;                                        // [1 + slice / 32 + 1]: bit of token i at 32 + i
    uint32_t *bidx = bits + a.slice / 32 + 2;                               // [slice / 2]: 16 bits a token, list entry + 1
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = int(cluster_ctarank());
    const int b = blockIdx.y, t0 = int(blockIdx.z) * a.range;
    cluster_arrive_relaxed();  // waited for before the first store into another CTA's memory
    pdl_wait();
    pdl_trigger();

    const int64_t nw64 = a.new_lens ? int64_t(__ldcg(a.new_lens + b)) + a.new_add : a.T;
    const int32_t L0 = a.lens ? __ldcg(a.lens + b) : 0;
    const bool ok = nw64 >= 0 && nw64 <= a.T && L0 >= 0 && L0 <= a.cap;
    const int nw = ok ? int(nw64) : 0;
    const int t1 = min(min(t0 + a.range, a.T), nw);  // positions of this cluster that have logits
    if (rank == 0 && tid == 0 && t0 == 0 && a.status) a.status[b] = ok ? SWITCHSD_ROW_OK : SWITCHSD_ROW_BAD_LEN;
    const float rep = a.rep ? __ldcg(a.rep + b) : 1.f, freq = a.freq ? __ldcg(a.freq + b) : 0.f, pres = a.pres ? __ldcg(a.pres + b) : 0.f;
    const bool penal = rep != 1.f || freq != 0.f || pres != 0.f;
    const int32_t v0 = rank * a.slice, v1 = min(a.V, v0 + a.slice);
    const int nv = max(0, v1 - v0);

    if (t0 < t1) {
        // --- counts, biases, the map of what is special ---------------------------------------------------------
        for (int i = tid; i < a.slice + a.slice / 32 + 2 + (a.nbias ? a.slice / 2 : 0); i += kLogitThreads) smem[i] = 0;
        const int ndraft = a.draft ? t1 - 1 : 0;  // draft tokens that some position here has behind it
        __syncthreads();
        if (penal) {
            const int32_t *x = a.ctx + size_t(b) * size_t(a.cap);
            const int32_t first = a.prompt ? __ldcg(a.prompt + b) : 0;
            for (int i = 4 * tid; i < L0; i += 4 * kLogitThreads) {
                const int4 r = __ldcg(reinterpret_cast<const int4 *>(x + i));
                const int32_t id[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t at = uint32_t(id[e]) - uint32_t(v0);
                    if (i + e < L0 && id[e] >= 0 && at < uint32_t(nv)) {
                        if (i + e >= first)
                            atomicAdd(&cnt[at], 1u);
                        else
                            atomicOr(&cnt[at], kSeen);
                    }
                }
            }
            for (int i = tid; i < ndraft; i += kLogitThreads) {
                const int32_t id = __ldcg(a.draft + size_t(b) * a.draft_stride + i);
                const uint32_t at = uint32_t(id) - uint32_t(v0);
                if (id >= 0 && at < uint32_t(nv)) atomicOr(&cnt[at], kInDraft);
            }
        }
        for (int i = tid; i < a.nbias; i += kLogitThreads) {
            const int32_t id = __ldcg(a.bias_ids + size_t(b) * a.nbias + i);
            const uint32_t at = uint32_t(id) - uint32_t(v0);
            if (id < 0 || at >= uint32_t(nv)) continue;
            // the last entry that names the token: a maximum of 16 bits, whatever the order of the threads
            const int sh = 16 * int(at & 1);
            uint32_t old = bidx[at >> 1];
            while (((old >> sh) & 0xffffu) < uint32_t(i + 1)) {
                const uint32_t seen = atomicCAS(&bidx[at >> 1], old, (old & ~(0xffffu << sh)) | (uint32_t(i + 1) << sh));
                if (seen == old) break;
                old = seen;
            }
        }
        __syncthreads();
        for (int i = warp; i < a.slice / 32; i += kLogitWarps) {
            const int at = 32 * i + lane;
            const bool sp = cnt[at] != 0 || (a.nbias && ((bidx[at >> 1] >> (16 * (at & 1))) & 0xffffu));
            const uint32_t m = __ballot_sync(kFull, sp);
            if (lane == 0) bits[1 + i] = m;
        }
        __syncthreads();

        // --- the positions --------------------------------------------------------------------------------------
        for (int t = t0; t < t1; ++t) {
            const elem *row = reinterpret_cast<const elem *>(a.logits) + int64_t(b) * a.sb + int64_t(t) * a.st + v0;
            elem *out = a.out ? reinterpret_cast<elem *>(a.out) + int64_t(b) * a.ob + int64_t(t) * a.ot + v0 : nullptr;
            const uint32_t *mask = a.mask ? a.mask + (size_t(b) * a.T + t) * a.mask_words : nullptr;
            const int mis = int((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(elem));
            const bool vec_out = out && ((reinterpret_cast<uintptr_t>(out) & 15) / sizeof(elem)) == size_t(mis);
            float best = -INFINITY;
            int32_t best_id = -1;
            const int nq = (nv + mis + N - 1) / N;
            for (int q = tid; q < nq; q += kLogitThreads) {
                const int e0 = q * N - mis;  // first element's place in the slice, negative in the first vector
                const bool whole = e0 >= 0 && e0 + N <= nv;
                elem v[N];
                if (whole) {
                    *reinterpret_cast<uint4 *>(v) = *reinterpret_cast<const uint4 *>(row + e0);
                } else {
#pragma unroll
                    for (int i = 0; i < N; ++i) v[i] = e0 + i >= 0 && e0 + i < nv ? row[e0 + i] : elem(0);
                }
                const int bit = e0 + 32;
                const uint32_t sp = __funnelshift_r(bits[bit >> 5], bits[min((bit >> 5) + 1, a.slice / 32 + 1)], bit & 31);
                uint32_t allow = 0xffffffffu;
                if (mask) {
                    const int ab = v0 + max(e0, 0), w = ab >> 5;
                    allow = __funnelshift_r(mask[w], mask[min(w + 1, a.mask_words - 1)], ab & 31) << (max(e0, 0) - e0);
                }
                float x[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    x[i] = E::get(v[i]);
                    if ((sp >> i) & 1) {
                        const int at = e0 + i;
                        if (at >= 0 && at < nv) {
                            const uint32_t c = cnt[at];
                            uint32_t extra = 0;
                            if (c & kInDraft)
                                for (int d = 0; d < t; ++d) extra += __ldcg(a.draft + size_t(b) * a.draft_stride + d) == v0 + at;
                            const uint32_t m = (c & kCount) + extra;
                            if ((c & kSeen) || m) x[i] = x[i] > 0.f ? __fdiv_rn(x[i], rep) : __fmul_rn(x[i], rep);
                            if (m) x[i] = __fsub_rn(__fsub_rn(x[i], __fmul_rn(freq, float(m))), pres);
                            if (a.nbias) {
                                const uint32_t k = (bidx[at >> 1] >> (16 * (at & 1))) & 0xffffu;
                                if (k) x[i] = __fadd_rn(x[i], __ldcg(a.bias + size_t(b) * a.nbias + k - 1));
                            }
                        }
                    }
                    if (!((allow >> i) & 1)) x[i] = -INFINITY;
                    if (x[i] > best && e0 + i >= 0 && e0 + i < nv) {
                        best = x[i];
                        best_id = v0 + e0 + i;
                    }
                }
                if (out) {
#pragma unroll
                    for (int i = 0; i < N; ++i) v[i] = E::put(x[i]);
                    if (whole && vec_out) {
                        *reinterpret_cast<uint4 *>(out + e0) = *reinterpret_cast<uint4 *>(v);
                    } else {
#pragma unroll
                        for (int i = 0; i < N; ++i)
                            if (e0 + i >= 0 && e0 + i < nv) out[e0 + i] = v[i];
                    }
                }
            }
            const uint64_t key = warp_max_u64(best_key(best, best_id));
            if (lane == 0) s_best[t - t0][warp] = key;
        }
    }
    __syncthreads();
    cluster_wait_acquire();
    if (t0 < t1) {
        for (int i = tid; i < t1 - t0; i += kLogitThreads) {
            uint64_t key = 0;
#pragma unroll
            for (int w = 0; w < kLogitWarps; ++w) key = s_best[i][w] > key ? s_best[i][w] : key;
            asm volatile("st.shared::cluster.u64 [%0], %1;\n" ::"r"(map_to_rank(&s_part[rank][i], 0)), "l"(key) : "memory");
        }
    }
    cluster_arrive_release();
    cluster_wait_acquire();
    if (rank == 0 && a.argmax) {
        for (int t = t0 + tid; t < min(t0 + a.range, a.T); t += kLogitThreads) {
            uint64_t key = 0;
            if (t < t1)
#pragma unroll
                for (int p = 0; p < kLogitParts; ++p) key = s_part[p][t - t0] > key ? s_part[p][t - t0] : key;
            a.argmax[size_t(b) * a.T + t] = key ? int32_t(~uint32_t(key)) : -1;
        }
    }
}

// Rows of the mask, padded: bytes of shared memory for a slice.
static size_t logits_smem(int32_t slice, int32_t nbias) {
    return (size_t(slice) + size_t(slice / 32) + 2 + (nbias ? size_t(slice) / 2 : 0)) * 4;
}

template <int DT>
static cudaError_t launch_logits(const LogitArgs &a, int B, int ranges, cudaStream_t s) {
    static bool attr_done[64] = {false};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_done[dev]) {
        e = cudaFuncSetAttribute(logits_kernel<DT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 int(logits_smem((SWITCHSD_VMAX / kLogitParts + 63) / 64 * 64, 1)));
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_done[dev] = true;
    }
    return launch_pdl(logits_kernel<DT>, dim3(kLogitParts, unsigned(B), unsigned(ranges)), dim3(kLogitThreads), logits_smem(a.slice, a.nbias), s,
                      unsigned(kLogitParts), a);
}

}  // namespace switchsd

using namespace switchsd;

extern "C" int switchsd_logits(const switchsd_logits_params *p) {
    if (!p || !p->logits || (!p->out && !p->argmax)) return SWITCHSD_ERR_ARG;
    if (p->dtype != SWITCHSD_BF16 && p->dtype != SWITCHSD_F16 && p->dtype != SWITCHSD_F32) return SWITCHSD_ERR_ARG;
    const uintptr_t size = p->dtype == SWITCHSD_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(p->logits) % size || reinterpret_cast<uintptr_t>(p->out) % size) return SWITCHSD_ERR_ARG;
    if ((p->ctx_tokens == nullptr) != (p->ctx_lens == nullptr) || (reinterpret_cast<uintptr_t>(p->ctx_tokens) & 15)) return SWITCHSD_ERR_ARG;
    if (p->nbias < 0 || (p->nbias > 0 && (!p->bias_ids || !p->bias))) return SWITCHSD_ERR_ARG;
    if (p->B < 1 || p->B > 65535 || p->T < 1 || p->V < 1 || p->V > SWITCHSD_VMAX || p->nbias > SWITCHSD_BIAS_MAX) return SWITCHSD_ERR_SHAPE;
    if (p->ctx_tokens && (p->cap < 4 || p->cap % 4 != 0 || p->cap >= (1 << 30))) return SWITCHSD_ERR_SHAPE;
    if (p->draft && p->T > 1 && p->draft_stride < p->T - 1) return SWITCHSD_ERR_SHAPE;
    if (p->mask && p->mask_words < (p->V + 31) / 32) return SWITCHSD_ERR_SHAPE;
    if (p->stride_b < 0 || p->stride_t < 0 || p->out_stride_b < 0 || p->out_stride_t < 0) return SWITCHSD_ERR_ARG;
    LogitArgs a;
    a.logits = static_cast<const uint8_t *>(p->logits);
    a.out = static_cast<uint8_t *>(p->out);
    a.sb = p->stride_b;
    a.st = p->stride_t;
    a.ob = p->out_stride_b;
    a.ot = p->out_stride_t;
    a.ctx = p->ctx_tokens;
    a.lens = p->ctx_lens;
    a.draft = p->T > 1 ? p->draft : nullptr;
    a.new_lens = p->new_lens;
    a.prompt = p->prompt_lens;
    a.bias_ids = p->bias_ids;
    a.rep = p->rep;
    a.freq = p->freq;
    a.pres = p->pres;
    a.bias = p->bias;
    a.mask = reinterpret_cast<const uint32_t *>(p->mask);
    a.argmax = p->argmax;
    a.status = p->status;
    a.T = p->T;
    a.V = p->V;
    a.cap = p->ctx_tokens ? p->cap : 0;
    a.draft_stride = p->draft_stride;
    a.new_add = p->new_add;
    a.nbias = p->nbias;
    a.mask_words = p->mask_words;
    a.slice = ((p->V + kLogitParts - 1) / kLogitParts + 63) / 64 * 64;
    // enough clusters for the chip, as few positions each as that takes (every cluster counts its row's context)
    const int want = std::max(1, 152 * 2 / (kLogitParts * p->B));
    a.range = std::min(kLogitRange, std::max(1, (p->T + want - 1) / want));
    const int ranges = (p->T + a.range - 1) / a.range;
    if (ranges > 65535) return SWITCHSD_ERR_SHAPE;
    cudaStream_t s = static_cast<cudaStream_t>(p->stream);
    const cudaError_t e = p->dtype == SWITCHSD_F32    ? launch_logits<SWITCHSD_F32>(a, p->B, ranges, s)
                          : p->dtype == SWITCHSD_F16 ? launch_logits<SWITCHSD_F16>(a, p->B, ranges, s)
                                                     : launch_logits<SWITCHSD_BF16>(a, p->B, ranges, s);
    return e == cudaSuccess ? SWITCHSD_OK : SWITCHSD_ERR_CUDA;
}
