// logprobs.cu -- switchsd_logprobs: log probabilities of given tokens, entropies and top alternatives.
//
// One pass.  A CTA (or a cluster of up to 8 where there are few positions) reads a position's logits once.  A thread keeps,
// relative to its running maximum m and with z = (l - m) / temperature, S = sum e^z and W = sum e^z z; a larger m scales both
// (W also loses what z gained).  The threads' meet in a tree; then lse = m / temperature + ln S, and the entropy is
// ln S - W / S.
//
// Top alternatives.  Of the first batch of loads (and again of the first four) the largest logit of every group of threads is
// known, and the k-th largest of those 128 is a bound that k of the CTA's logits reach: what lies below is no alternative.
// The few that do not go, one by one, into their warp's list, sorted over its lanes, whose k-th raises the warp's own bound.
// The lists (of all CTAs) are ranked by counting at the end.  A batch is looked at again only where its largest logit, which
// the sums want anyway, reaches the bound.
//
// Bound (128,256 tokens).  f32 logits: memory, 2048 positions in 153 us (103 % of a copy's rate, all of it reads), 164 with
// five alternatives.  16-bit ones: instructions, ten a logit with five alternatives: 2048 positions 92 us (84 %) without, with 5 /
// 20 / 32 alternatives 102 / 132 / 151; 8192 positions with five 352 (88 %).  One position (f32): 6.8 us, 11.6 with 20
// alternatives: a chain of loads, the bound, the lists, two rankings and two cluster barriers.
//
// What made the difference: one multiply-add a logit for z and packed sums (662 -> 511 us of the 8192 positions), a bound of
// 128 groups (of a warp's maxima: 40 logits a warp passed it), a second bound (460 -> 445), smaller CTAs, and a batch that
// lies inside the row loaded from one address (409 -> 352).  Batches of two vectors a thread instead of four: 497 against 445;
// three batches in shared memory instead of two: 467 against 436.
#include "sampling.cuh"

#include <algorithm>

namespace switchsd {

// Threads of a CTA.  Few positions are clusters of large CTAs (one position: 12.8 us, as a single CTA 35).  More are a CTA
// each: large ones while an SM has no more than three (450 positions with 512 / 256 / 128 threads: 35 / 38 / 39 us), smaller
// ones beyond, so that some of an SM's wait for each other or for their sums while others stream (1088 positions: 37 / 35 / 54;
// 3648: 232 / 198 / 191).  f32 logits want the loads in flight that 256 threads have (3648: 297 / 272 / 309).
constexpr int kProbMost = 128, kProbMany = 256, kProbFew = 512;
constexpr int kProbFlight = 4;          // vectors of a thread that are worked on together
constexpr int kProbRing = 2;            // batches of them in shared memory, or on their way there
// More alternatives than these have a bound again whenever twice as much has been read (2048 positions, bf16, 32 of them: 151
// instead of 178 us; 12: 118, 123; 5: 106 instead of 102), but where positions are few (20 of one: 13.1 instead of 12.0).
constexpr int kProbOften = 8;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kGone = -200.f;         // binary logarithm of a weight that binary32 does not have

struct ProbArgs {
    const void *logits;
    int64_t sb, st;
    const int32_t *new_lens, *tokens;
    const float *temperature;
    float *logprob, *prob, *entropy, *lse;
    int32_t *top_ids;
    float *top_logprobs;
    int32_t *status;
    int32_t T, V, K, top, new_add, tokens_stride;
};

// max, sum of weights, sum of weights times their binary logarithms
struct Sums {
    float m, s, w;
    __device__ void scale_to(float top, float c2) {  // top >= m
        const float d = fmaxf((m - top) * c2, kGone), f = exp2_fast(d);  // (the clamp also takes -inf - -inf)
        w = f * fmaf(s, d, w);
        s *= f;
        m = top;
    }
    __device__ void add(Sums o, float c2) {
        const float top = fmaxf(m, o.m);
        scale_to(top, c2);
        o.scale_to(top, c2);
        s += o.s;
        w += o.w;
    }
};

// Places in the order of floats (0 of what is not a number, -inf and what is not there come first); -0 and 0 share one.
__device__ __forceinline__ uint32_t place_of(float v) {
    const uint32_t u = __float_as_uint(v + 0.f);
    return v == v ? (u & 0x80000000u ? ~u : u | 0x80000000u) : 0u;
}
__device__ __forceinline__ float at_place(uint32_t p) {
    return p == 0 ? -INFINITY : __uint_as_float(p & 0x80000000u ? p & 0x7fffffffu : ~p);
}
// A bound that k of a warp's 128 numbers (four a lane, by their places) reach, as large as 20 bits can say, or
// (soon) as soon as the others do not; the same for all lanes.
__device__ __forceinline__ float kth_largest(const uint32_t (&p)[4], int k, bool soon) {
    uint32_t bound = 0;
#pragma unroll 1
    for (uint32_t bit = 0x80000000u; bit >= 0x1000u; bit >>= 1) {
        const uint32_t trial = bound | bit;
        int n = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) n += __popc(__ballot_sync(kFull, p[i] >= trial));
        if (n >= k) bound = trial;
        if (soon && n == k) break;
    }
    return bound > 0x007fffffu ? at_place(bound) : -INFINITY;  // (the place of -inf)
}

__device__ __forceinline__ bool before(float v, int32_t i, float w, int32_t j) { return v > w || (v == w && i < j); }

// A warp's 32 best (value, token) pairs, a lane each, in order.
struct WarpList {
    float v = -INFINITY, last = -INFINITY;  // this lane's, and the k-th
    int32_t id = 0x7fffffff;
    // The lanes' pairs, those with x > last (or the first of equal ones).
    __device__ __forceinline__ void insert(float x, int32_t token, int k) {
        uint32_t todo = __ballot_sync(kFull, x > last || (x == last && x > -INFINITY));
        const int lane = threadIdx.x & 31;
        while (todo) {
            const int src = __ffs(int(todo)) - 1;
            todo &= todo - 1;
            const float nv = __shfl_sync(kFull, x, src);
            const int32_t ni = __shfl_sync(kFull, token, src);
            const int place = __popc(__ballot_sync(kFull, before(v, id, nv, ni)));
            const float uv = __shfl_up_sync(kFull, v, 1);
            const int32_t ui = __shfl_up_sync(kFull, id, 1);
            if (lane >= place) {
                v = lane == place ? nv : uv;
                id = lane == place ? ni : ui;
            }
        }
        last = __shfl_sync(kFull, v, k - 1);
    }
};

// The first k of n (value, token) pairs in `v`, `id`, in order, to `out_v`, `out_id` (the same for all threads of the CTA):
// eight threads count those before a pair.
__device__ __forceinline__ void rank_pairs(const float *v, const int32_t *id, int n, int k, float *out_v, int32_t *out_id) {
    const int of = threadIdx.x & 7;
    for (int i0 = 0; i0 < n; i0 += int(blockDim.x) / 8) {
        const int i = i0 + int(threadIdx.x) / 8;
        const float x = i < n ? v[i] : INFINITY;
        const int32_t t = i < n ? id[i] : -1;
        int rank = 0;
        if (i < n)
            for (int j = of; j < n; j += 8) rank += before(v[j], id[j], x, t);
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) rank += __shfl_xor_sync(kFull, rank, o);
        if (of == 0 && i < n && rank < k) {
            out_v[rank] = x;
            out_id[rank] = t;
        }
    }
}

template <int DT, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) logprobs_kernel(const ProbArgs a, int parts) {
    using Row = LogitRow<DT>;
    constexpr int kProbThreads = THREADS, kProbWarps = THREADS / kWarp;
    constexpr int kGroup = THREADS / 128;                   // threads whose largest logit is looked at as one
    constexpr int P = Row::P, F = kProbFlight;
    extern __shared__ __align__(16) uint4 s_ring[];         // [kProbRing][F][threads], a thread's own
    __shared__ float s_group[128];
    __shared__ float s_bound;
    __shared__ Sums s_sums[kProbWarps], s_all;
    __shared__ float s_value[512], s_top[32];  // of the CTA's warps, or of the cluster's CTAs (8 at the most)
    __shared__ int32_t s_id[512], s_top_id[32];
    __shared__ int s_n, s_n_top;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int t = int(blockIdx.x) / parts, part = int(blockIdx.x) - t * parts, b = blockIdx.y;
    pdl_wait();
    pdl_trigger();
    const int64_t nw64 = a.new_lens ? int64_t(__ldcg(a.new_lens + b)) + a.new_add : a.T;
    const bool ok = nw64 >= 0 && nw64 <= a.T;
    if (a.status && t == 0 && part == 0 && tid == 0) a.status[b] = ok ? SWITCHSD_ROW_OK : SWITCHSD_ROW_BAD_LEN;
    const int64_t at = int64_t(b) * a.T + t;
    if (!ok || t >= nw64) {
        if (part == 0) {
            if (tid == 0) {
                if (a.entropy) a.entropy[at] = 0.f;
                if (a.lse) a.lse[at] = -INFINITY;
                if (t < a.K) {
                    if (a.logprob) a.logprob[int64_t(b) * a.K + t] = -INFINITY;
                    if (a.prob) a.prob[int64_t(b) * a.K + t] = 0.f;
                }
            }
            if (tid < a.top) {
                if (a.top_ids) a.top_ids[at * a.top + tid] = -1;
                if (a.top_logprobs) a.top_logprobs[at * a.top + tid] = -INFINITY;
            }
        }
        return;
    }
    const float temperature = a.temperature ? __ldcg(a.temperature + b) : 1.f;
    const bool greedy = temperature == 0.f;
    const float c2 = greedy ? 1.f : fminf(kLog2e / temperature, 3e38f);
    const int k = a.top > 0 ? a.top : greedy ? 1 : 0;  // alternatives to find
    const Row row(a.logits, b * a.sb + t * a.st, a.V);
    const int32_t per = (row.vectors + parts - 1) / parts, begin = part * per, end = min(begin + per, row.vectors);
    if (tid == 0) s_n = s_n_top = 0;

    Sums sums{-INFINITY, 0.f, 0.f};
    float bound = -INFINITY;                   // of the CTA: k logits reach it
    WarpList list;
    float most = -INFINITY;                    // this thread's largest logit
    int batch = 0;
    uint4 x[F], *slot = s_ring + tid;          // of the batch that is next
#pragma unroll
    for (int r = 0; r < kProbRing; ++r) {
        row.template fetch<F>(slot + r * F * kProbThreads, kProbThreads, begin + tid + r * F * kProbThreads, kProbThreads, end);
        cp_async_commit();
    }
    for (int32_t base = begin; base < end; base += kProbThreads * F) {
        cp_async_wait<kProbRing - 1>();
#pragma unroll
        for (int i = 0; i < F; ++i) x[i] = slot[i * kProbThreads];
        row.template fetch<F>(slot, kProbThreads, base + tid + kProbRing * F * kProbThreads, kProbThreads, end);
        cp_async_commit();
        slot = slot == s_ring + tid + (kProbRing - 1) * F * kProbThreads ? s_ring + tid : slot + F * kProbThreads;
        const float top = Row::largest(x);
        most = fmaxf(most, top);
        // (again when there is four times as much to go by: half of what passed the first bound does not pass the second)
        if (k > 0 && (batch & (batch + 1)) == 0 && (batch == 0 || batch == 3 || (k > kProbOften && THREADS != kProbFew))) {
            float g = most;
#pragma unroll
            for (int o = 1; o < kGroup; o <<= 1) g = fmaxf(g, __shfl_xor_sync(kFull, g, o));
            if (lane % kGroup == 0) s_group[tid / kGroup] = g;
            __syncthreads();
            if (warp == 0) {
                const uint32_t p[4] = {place_of(s_group[lane]), place_of(s_group[lane + 32]), place_of(s_group[lane + 64]), place_of(s_group[lane + 96])};
                g = kth_largest(p, k, THREADS == kProbFew);  // (where latency counts)
                if (lane == 0) s_bound = g;
            }
            __syncthreads();
            bound = s_bound;
        }
        ++batch;
        if (top > sums.m) sums.scale_to(top, c2);
        // Where a logit at kLow has no weight, what lies below (-inf, NaN) is taken for it, and z is one multiply-add off the
        // reference m c2, whose rounding is put right at the batch's end.
        const float ref = sums.m * c2;
        if ((sums.m - Row::kLow) * c2 >= -kGone && fabsf(ref) < 1e30f && c2 < 1e6f) {
            const float off = fmaf(sums.m, c2, -ref);
            const uint64_t c = pair_of(c2, c2), r = pair_of(-ref, -ref);
            uint64_t s2[2] = {0, 0}, w2[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < F; ++i) {
                float v[P];
                Row::widen(Row::raised(x[i]), v);
#pragma unroll
                for (int e = 0; e < P; e += 2) {
                    const uint64_t z = fma_pair(pair_of(v[e], v[e + 1]), c, r);
                    const float2 y = halves_of(z);
                    const uint64_t p = pair_of(exp2_fast(y.x), exp2_fast(y.y));
                    s2[(e >> 1) & 1] = add_pair(s2[(e >> 1) & 1], p);
                    w2[(e >> 1) & 1] = fma_pair(p, z, w2[(e >> 1) & 1]);
                }
            }
            const float2 sp = halves_of(add_pair(s2[0], s2[1])), wp = halves_of(add_pair(w2[0], w2[1]));
            const float f = exp2_fast(-off), part_s = sp.x + sp.y;
            sums.s = fmaf(part_s, f, sums.s);
            sums.w = fmaf(fmaf(-off, part_s, wp.x + wp.y), f, sums.w);
        } else {
            float s2 = 0.f, w2 = 0.f;
#pragma unroll
            for (int i = 0; i < F; ++i) {
                float v[P];
                Row::widen(x[i], v);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    const float y = fmaxf((v[e] - sums.m) * c2, kGone), p = exp2_fast(y);  // (NaN: no weight)
                    s2 += p;
                    w2 = fmaf(p, y, w2);
                }
            }
            sums.s += s2;
            sums.w += w2;
        }
        if (k > 0 && __any_sync(kFull, top >= bound && top > list.last)) {
#pragma unroll
            for (int i = 0; i < F; ++i) {
                const uint4 one[1] = {x[i]};
                const float best = Row::largest(one);
                if (!__any_sync(kFull, best >= bound && best > list.last)) continue;
                float v[P];
                Row::widen(x[i], v);
                uint32_t mask = 0;
#pragma unroll
                for (int e = 0; e < P; ++e) mask |= uint32_t(v[e] >= bound && v[e] > list.last) << e;
                const int32_t from = row.token(base + tid + i * kProbThreads);
#pragma unroll 1
                while (__any_sync(kFull, mask != 0)) {
                    const int e = __ffs(int(mask)) - 1;  // (-1: nothing)
                    mask &= mask - 1;
                    float y = -INFINITY;
#pragma unroll
                    for (int j = 0; j < P; ++j) y = e == j ? v[j] : y;
                    list.insert(y, from + e, k);
                }
            }
        }
    }

    // --- the CTA's ------------------------------------------------------------------------------------------------
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        sums.add(Sums{__shfl_xor_sync(kFull, sums.m, o), __shfl_xor_sync(kFull, sums.s, o), __shfl_xor_sync(kFull, sums.w, o)}, c2);
    if (lane == 0) s_sums[warp] = sums;
    __syncthreads();
    if (k > 0) {
        const bool has = lane < k && list.v >= bound && list.v > -INFINITY;
        const uint32_t those = __ballot_sync(kFull, has);
        int from = 0;
        if (lane == 0 && those) from = atomicAdd(&s_n, __popc(those));
        from = __shfl_sync(kFull, from, 0) + __popc(those & ((1u << lane) - 1));
        if (has) {
            s_value[from] = list.v;
            s_id[from] = list.id;
        }
        __syncthreads();
        rank_pairs(s_value, s_id, s_n, k, s_top, s_top_id);
    }
    if (warp == 0) {
        sums = lane < kProbWarps ? s_sums[lane] : Sums{-INFINITY, 0.f, 0.f};
#pragma unroll
        for (int o = kProbWarps / 2; o > 0; o >>= 1)
            sums.add(Sums{__shfl_xor_sync(kFull, sums.m, o), __shfl_xor_sync(kFull, sums.s, o), __shfl_xor_sync(kFull, sums.w, o)}, c2);
        if (lane == 0) {
            s_all = sums;
            s_n_top = min(s_n, k);
        }
    }
    __syncthreads();

    // --- the cluster's --------------------------------------------------------------------------------------------
    if (parts > 1) {
        cluster_arrive_release();
        cluster_wait_acquire();
        if (part == 0) {
            if (warp == 0) {
                sums = Sums{-INFINITY, 0.f, 0.f};
                if (lane < parts) sums = Sums{remote_float(&s_all.m, lane), remote_float(&s_all.s, lane), remote_float(&s_all.w, lane)};
#pragma unroll
                for (int o = 4; o > 0; o >>= 1)
                    sums.add(Sums{__shfl_xor_sync(kFull, sums.m, o), __shfl_xor_sync(kFull, sums.s, o), __shfl_xor_sync(kFull, sums.w, o)}, c2);
            }
            if (k > 0) {  // part tid / 32's list, place tid % 32
                __syncthreads();
                if (tid == 0) s_n = 0;
                __syncthreads();
                if (warp < parts && lane < int(remote_word(&s_n_top, warp))) {
                    const int i = atomicAdd(&s_n, 1);
                    s_value[i] = remote_float(&s_top[lane], warp);
                    s_id[i] = int32_t(remote_word(&s_top_id[lane], warp));
                }
                __syncthreads();
                rank_pairs(s_value, s_id, s_n, k, s_top, s_top_id);  // (all have read this CTA's list)
            }
            __syncthreads();
            if (tid == 0) {
                s_all = sums;
                s_n_top = min(s_n, k);
            }
            __syncthreads();
        }
        cluster_arrive_release();  // the others' shared memory is read until here
        cluster_wait_acquire();
        if (part != 0) return;
    }
    const float m = s_all.m, log_s = logf(s_all.s);
    const bool bad = !(temperature >= 0.f && temperature < INFINITY) || (m == INFINITY && !greedy), none = m == -INFINITY;
    const float nan = __int_as_float(0x7fc00000);
    auto logprob_of = [&](float l, int32_t id) {
        if (!(l > -INFINITY)) return -INFINITY;
        if (bad) return nan;
        if (greedy) return id == s_top_id[0] ? 0.f : -INFINITY;
        return (l - m) / temperature - log_s;
    };
    if (tid == 0) {
        const bool bad_t = !(temperature >= 0.f && temperature < INFINITY);
        if (a.lse) a.lse[at] = bad_t ? nan : none || greedy || m == INFINITY ? m : m / temperature + log_s;
        if (a.entropy) a.entropy[at] = none || greedy ? 0.f : bad ? nan : fmaxf(0.f, log_s - s_all.w / s_all.s * kLn2);
        if (t < a.K) {
            const int32_t token = __ldcg(a.tokens + int64_t(b) * a.tokens_stride + t);
            const float lp = uint32_t(token) < uint32_t(a.V) ? logprob_of(row[token], token) : -INFINITY;
            if (a.logprob) a.logprob[int64_t(b) * a.K + t] = lp;
            if (a.prob) a.prob[int64_t(b) * a.K + t] = expf(lp);
        }
    }
    if (tid < a.top) {
        const bool there = tid < s_n_top;
        if (a.top_ids) a.top_ids[at * a.top + tid] = there ? s_top_id[tid] : -1;
        if (a.top_logprobs) a.top_logprobs[at * a.top + tid] = there ? logprob_of(s_top[tid], s_top_id[tid]) : -INFINITY;
    }
}

template <int DT, int THREADS>
static cudaError_t launch_logprobs(const ProbArgs &a, int32_t B, int parts, cudaStream_t s) {
    static bool attr_done[64] = {false};
    constexpr int kSmem = kProbRing * kProbFlight * THREADS * 16;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_done[dev]) {
        e = cudaFuncSetAttribute(logprobs_kernel<DT, THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_done[dev] = true;
    }
    const dim3 grid(unsigned(parts) * unsigned(a.T), unsigned(B));
    return launch_pdl(logprobs_kernel<DT, THREADS>, grid, dim3(THREADS), size_t(kSmem), s, parts > 1 ? unsigned(parts) : 0u, a, parts);
}
template <int DT>
static cudaError_t launch_logprobs(const ProbArgs &a, int32_t B, cudaStream_t s) {
    const int64_t sms = sm_count(), rows = int64_t(B) * a.T;
    if (sms == 0) return cudaErrorInvalidDevice;
    const int parts = parts_of(rows, (int64_t(a.V) + LogitRow<DT>::P - 1) / LogitRow<DT>::P, kProbFew, 2 * sms);
    if (rows <= 3 * sms) return launch_logprobs<DT, kProbFew>(a, B, parts, s);
    if (DT == SWITCHSD_F32 || rows <= 12 * sms) return launch_logprobs<DT, kProbMany>(a, B, 1, s);
    return launch_logprobs<DT, kProbMost>(a, B, 1, s);
}

}  // namespace switchsd

using namespace switchsd;

extern "C" int switchsd_logprobs(const switchsd_logprobs_params *p) {
    if (!p || !p->logits) return SWITCHSD_ERR_ARG;
    if (p->dtype != SWITCHSD_BF16 && p->dtype != SWITCHSD_F16 && p->dtype != SWITCHSD_F32) return SWITCHSD_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(p->logits) % (p->dtype == SWITCHSD_F32 ? 4 : 2)) return SWITCHSD_ERR_ARG;
    const bool of_tokens = p->logprob || p->prob, of_top = p->top_ids || p->top_logprobs;
    if (!of_tokens && !of_top && !p->entropy && !p->lse) return SWITCHSD_ERR_ARG;
    if (of_tokens && (p->K < 1 || !p->tokens)) return SWITCHSD_ERR_ARG;
    if (of_top && p->top < 1) return SWITCHSD_ERR_ARG;
    if ((p->stride_b < 0 && p->B > 1) || (p->stride_t < 0 && p->T > 1)) return SWITCHSD_ERR_ARG;
    if (p->B < 1 || p->B > 65535 || p->T < 1 || p->T > 262140 || p->V < 1 || p->V > SWITCHSD_VMAX || p->K < 0 || p->K > p->T || p->top < 0 ||
        p->top > SWITCHSD_TOP_MAX || (of_tokens && p->tokens_stride < p->K))
        return SWITCHSD_ERR_SHAPE;
    ProbArgs a;
    a.logits = p->logits;
    a.sb = stride_of(p->stride_b, p->B);
    a.st = stride_of(p->stride_t, p->T);
    a.new_lens = p->new_lens;
    a.tokens = p->tokens;
    a.temperature = p->temperature;
    a.logprob = p->logprob;
    a.prob = p->prob;
    a.entropy = p->entropy;
    a.lse = p->lse;
    a.top_ids = p->top_ids;
    a.top_logprobs = p->top_logprobs;
    a.status = p->status;
    a.T = p->T;
    a.V = p->V;
    a.K = of_tokens ? p->K : 0;
    a.top = of_top ? p->top : 0;
    a.new_add = p->new_add;
    a.tokens_stride = p->tokens_stride;
    cudaStream_t s = static_cast<cudaStream_t>(p->stream);
    const cudaError_t e = p->dtype == SWITCHSD_F32   ? launch_logprobs<SWITCHSD_F32>(a, p->B, s)
                          : p->dtype == SWITCHSD_F16 ? launch_logprobs<SWITCHSD_F16>(a, p->B, s)
                                                     : launch_logprobs<SWITCHSD_BF16>(a, p->B, s);
    return e == cudaSuccess ? SWITCHSD_OK : SWITCHSD_ERR_CUDA;
}
