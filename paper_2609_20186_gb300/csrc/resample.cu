// resample.cu -- switchsd_resample: the token that the sampled verification appends.
//
// An exponential race: with E_v exponential variables, the largest w_v / E_v is v with probability w_v / sum w, so one pass
// over the one row of logits that counts decides, without a sum over the vocabulary.  The random bits are a function of
// the row's seed, the token's place in the context and v.
//
// Screening.  E = -ln(1 - x) is at least x, so v beats a score s only where x < w_v e^-s: a binary exponential and a
// comparison of the number's upper 23 bits, beside the bits themselves (two 64-bit products for two tokens).  s is the
// best score of the CTA so far, to begin with of one logit a thread; few tokens pass, and they alone are worked out, in
// binary32.  Where two scores are closer than its error, both are worked out in binary64, so the answer is that of
// binary64 throughout.  A drafter's distribution is read for the few only: w = max(0, p - q) is at most p.
#include "sampling.cuh"

namespace switchsd {

constexpr int kRaceThreads = 512;
constexpr int kRaceFlight = 4;          // vectors of a thread in flight
constexpr float kRaceLog2e = 1.4426950408889634f;

struct RaceArgs {
    const void *logits, *q_logits;
    int64_t sb, st, qb, qt;
    const float *lse, *q_lse, *temperature, *p, *q, *u;
    const int32_t *draft, *draft_len, *mode, *ctx_lens;
    const int64_t *seeds;
    int32_t *out, *status;
    int32_t T, V;
};

__device__ __forceinline__ uint64_t splitmix(uint64_t z) {  // the output function of splitmix64 (Steele, Lea and Flood, 2014)
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}
constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;

// Numbers in the order of floats (no NaN), for atomicMax.
__device__ __forceinline__ int32_t float_order(float v) {
    const int32_t i = __float_as_int(v);
    return i < 0 ? i ^ 0x7fffffff : i;
}
__device__ __forceinline__ float order_float(int32_t i) { return __int_as_float(i < 0 ? i ^ 0x7fffffff : i); }

// What a row's weights go by.
template <int DT>
struct Race {
    LogitRow<DT> l, q;
    uint64_t key;
    float temperature, lse, q_lse;
    int32_t skip;          // a token that has no weight, or -1
    bool residual, greedy;
    __device__ uint32_t bits(int32_t v) const {
        const uint64_t z = splitmix(key + (uint64_t(uint32_t(v) >> 1) + 1) * kGolden);
        return (v & 1) ? uint32_t(z >> 32) : uint32_t(z);
    }
    __device__ __noinline__ double exact(int32_t v) const {
        const double z = double(l[v]);
        if (greedy) return z;
        double y = z / double(temperature);
        if (residual) {
            const float zq = q[v];
            y -= double(lse);
            const double w = exp(y) - (zq > -INFINITY ? exp(double(zq) / double(temperature) - double(q_lse)) : 0.);
            if (!(w > 0.)) return -INFINITY;
            y = log(w);
        }
        return y - log(-log1p(-(double(bits(v)) + 0.5) * 0x1p-32));
    }
    // ln w - ln E of token v with logit z, -inf where it has no weight.
    __device__ float score(int32_t v, float z) const {
        if (!(z > -INFINITY) || v == skip) return -INFINITY;
        if (greedy) return z;
        float y = z / temperature;
        if (residual) {
            const float zq = q[v];
            if (zq > -INFINITY) {
                const float a = (zq - z) / temperature, b = q_lse - lse, d = a - b;  // ln(q / p)
                if (d > 0.0078125f + 1e-4f * (fabsf(a) + fabsf(b))) return -INFINITY;
                if (!(d < -0.0078125f - 1e-4f * (fabsf(a) + fabsf(b)))) return float(exact(v));  // p - q nearly cancels
                y += logf(-expm1f(d));
            }
            y -= lse;
        }
        const uint32_t r = bits(v);
        const float e = r < 0x80000000u ? -log1pf(-(float(r) + 0.5f) * 0x1p-32f) : -logf((float(~r) + 0.5f) * 0x1p-32f);
        return y - logf(e);
    }
    // How far binary32's score may be off, and binary64's of what is compared with it.
    __device__ float margin(float s) const { return greedy || fabsf(s) == INFINITY ? 0.f : (residual ? 4e-3f : 2e-5f) + 1e-6f * fabsf(s); }
};

template <int DT>
struct Best {
    float s = -INFINITY;
    int32_t v = -1;
    __device__ void consider(const Race<DT> &race, int32_t token, float z) {
        const float x = race.score(token, z);
        if (!(x > -INFINITY) || token == v) return;
        const float margin = race.margin(x);
        bool take = v < 0 || x > s + margin;
        if (!take && x >= s - margin) {
            const double mine = race.exact(token), other = race.exact(v);
            take = mine > other || (mine == other && token < v);
        }
        if (take) {
            s = x;
            v = token;
        }
    }
};

template <int DT>
__global__ void __launch_bounds__(kRaceThreads, 2) resample_kernel(const RaceArgs a, int parts) {
    using Row = LogitRow<DT>;
    constexpr int P = Row::P, F = kRaceFlight;
    __shared__ int32_t s_first, s_best, s_n;
    __shared__ int32_t s_list[kRaceThreads];
    __shared__ double s_exact[kRaceThreads];
    const int tid = threadIdx.x, part = blockIdx.x, b = blockIdx.y, k = a.T - 1;
    pdl_wait();
    pdl_trigger();
    const int32_t len = __ldcg(a.draft_len + b), ctx = __ldcg(a.ctx_lens + b);
    const bool ok = len >= 0 && len <= k && ctx >= 0;
    if (part == 0) {
        if (tid == 0 && a.status) a.status[b] = ok ? SWITCHSD_ROW_OK : SWITCHSD_ROW_BAD_LEN;
        if (!ok)
            for (int i = tid; i < a.T; i += kRaceThreads) a.out[int64_t(b) * a.T + i] = -1;
    }
    if (!ok) return;
    // --- the accepted length --------------------------------------------------------------------------------------
    if (tid == 0) {
        s_first = len;
        s_n = 0;
        s_best = float_order(-INFINITY);
    }
    __syncthreads();
    for (int i = tid; i < len; i += kRaceThreads) {
        const int64_t at = int64_t(b) * k + i;
        const float q = a.q ? __ldcg(a.q + at) : 1.f;
        if (!(__fmul_rn(__ldcg(a.u + at), q) < __ldcg(a.p + at))) {
            atomicMin(&s_first, i);
            break;
        }
    }
    __syncthreads();
    const int acc = s_first;
    if (part == 0)
        for (int i = tid; i < a.T; i += kRaceThreads)
            if (i != acc) a.out[int64_t(b) * a.T + i] = -1;
    // --- the weights ----------------------------------------------------------------------------------------------
    const bool drafted = acc < len, drafter = drafted && a.q_logits && !(a.mode && __ldcg(a.mode + b) == SWITCHSD_MODE_COPY);
    const Row row(a.logits, b * a.sb + acc * a.st, a.V);
    Race<DT> race{row, drafter ? Row(a.q_logits, b * a.qb + acc * a.qt, a.V) : row};
    race.key = splitmix(uint64_t(__ldcg(a.seeds + b)) + (uint64_t(ctx) + uint64_t(acc) + 1) * kGolden);
    race.temperature = a.temperature ? __ldcg(a.temperature + b) : 1.f;
    race.greedy = race.temperature == 0.f;
    race.residual = drafter && !race.greedy;
    race.lse = race.residual ? __ldcg(a.lse + int64_t(b) * a.T + acc) : 0.f;
    race.q_lse = race.residual ? __ldcg(a.q_lse + int64_t(b) * k + acc) : 0.f;
    race.skip = drafted && !drafter && !race.greedy ? __ldcg(a.draft + int64_t(b) * k + acc) : -1;
    const bool none = !(race.temperature >= 0.f && race.temperature < INFINITY) || race.lse != race.lse || race.q_lse != race.q_lse;
    const int32_t per = (row.vectors + parts - 1) / parts, begin = part * per, end = min(begin + per, row.vectors);
    const float c2 = fminf(kRaceLog2e / race.temperature, 3e38f);
    Best<DT> best;
    float top = -INFINITY;
    for (int round = 0; !none; ++round) {
        if (race.greedy) {
            for (int32_t j = begin + tid; j < end; j += kRaceThreads) {
                float x[P];
                Row::widen(row.load(j, end), x);
#pragma unroll
                for (int e = 0; e < P; ++e)
                    if (x[e] > best.s) {  // (ascending tokens)
                        best.s = x[e];
                        best.v = row.token(j) + e;
                    }
            }
        } else {
            const int32_t v0 = row.token(begin + tid) + (tid & (P - 1));
            if (begin + tid < end && uint32_t(v0) < uint32_t(a.V)) best.consider(race, v0, row[v0]);
            atomicMax(&s_best, float_order(best.s));
            __syncthreads();
            const float lse2 = race.lse * kRaceLog2e;
            for (int32_t base = begin + tid; base < end; base += kRaceThreads * F) {
                uint4 w[F];
#pragma unroll
                for (int i = 0; i < F; ++i) w[i] = row.load(base + i * kRaceThreads, end);
                // A lower bound of the best score, in binary logarithms, less what the test's own roundings may take.
                const float s = order_float(*static_cast<volatile int32_t *>(&s_best));
                const float s2 = (s - race.margin(s)) * kRaceLog2e;
                const float off = fabsf(s) < 1e30f ? 1e-3f + 4e-7f * (fabsf(s2) + fabsf(lse2)) - s2 - lse2 : INFINITY;
#pragma unroll 1
                for (int i = 0; i < F; ++i) {
                    const int32_t j = base + i * kRaceThreads;
                    if (j >= end) break;
                    float x[P];
                    Row::widen(w[0], x);
#pragma unroll
                    for (int o = 0; o < F - 1; ++o) w[o] = w[o + 1];
                    const int32_t from = row.token(j);
                    uint64_t n = race.key + (uint64_t(int64_t(from >> 1)) + 1) * kGolden;  // of the pair that `from` lies in
                    uint64_t z = splitmix(n);
                    uint32_t mask = 0;
                    auto test = [&](int e, uint32_t r) {
                        // 1 + (x rounded down to 23 bits) <= 1 + w e^-s
                        const float t = exp2f(fmaf(x[e], c2, off));
                        mask |= uint32_t(__uint_as_float(0x3f800000u | (r >> 9)) <= fmaf(t, 1.002f, 1.0000003f)) << e;
                    };
                    if (from & 1) {
#pragma unroll
                        for (int e = 0; e < P; e += 2) {
                            test(e, uint32_t(z >> 32));
                            z = splitmix(n += kGolden);
                            test(e + 1, uint32_t(z));
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < P; e += 2) {
                            if (e) z = splitmix(n += kGolden);
                            test(e, uint32_t(z));
                            test(e + 1, uint32_t(z >> 32));
                        }
                    }
                    while (mask) {
                        const int e = __ffs(int(mask)) - 1;
                        mask &= mask - 1;
                        const int32_t v = from + e;
                        if (uint32_t(v) >= uint32_t(a.V)) continue;
                        best.consider(race, v, row[v]);
                        atomicMax(&s_best, float_order(best.s));
                    }
                }
            }
        }
        // --- the best of all: those that binary32 does not tell from it, in binary64 ------------------------------
        if (race.greedy) atomicMax(&s_best, float_order(best.s));
        __syncthreads();
        top = order_float(s_best);
        if (parts > 1) {
            cluster_arrive_release();
            cluster_wait_acquire();
            for (int r = 0; r < parts; ++r) top = fmaxf(top, order_float(int32_t(remote_word(&s_best, r))));
        }
        if (top > -INFINITY || round == 1 || (!race.residual && race.skip < 0)) break;
        // nothing is left of w: once more with p
        if (parts > 1) {
            cluster_arrive_release();  // (all have read s_best)
            cluster_wait_acquire();
        }
        __syncthreads();
        race.residual = false;
        race.lse = race.q_lse = 0.f;
        race.skip = -1;
    }
    int32_t token = -1;
    if (top > -INFINITY) {
        if (best.v >= 0 && best.s >= top - 2.f * race.margin(top)) s_list[atomicAdd(&s_n, 1)] = best.v;
        __syncthreads();
        if (parts > 1) {
            cluster_arrive_release();
            cluster_wait_acquire();
        }
        if (part == 0) {
            double of_token = -INFINITY;
            int all = 0;
            for (int r = 0; r < parts; ++r) all += parts > 1 ? int(remote_word(&s_n, r)) : s_n;
            for (int r = 0; r < parts; ++r) {
                const int n = parts > 1 ? int(remote_word(&s_n, r)) : s_n;
                int32_t mine = -1;
                if (tid < n) {
                    mine = parts > 1 ? int32_t(remote_word(&s_list[tid], r)) : s_list[tid];
                    s_exact[tid] = all == 1 ? 0. : race.exact(mine);
                }
                __syncthreads();
                if (tid == 0)
                    for (int i = 0; i < n; ++i) {
                        const int32_t v = parts > 1 ? int32_t(remote_word(&s_list[i], r)) : s_list[i];
                        if (token < 0 || s_exact[i] > of_token || (s_exact[i] == of_token && v < token)) {
                            token = v;
                            of_token = s_exact[i];
                        }
                    }
                __syncthreads();
            }
        }
    }
    if (part == 0 && tid == 0) a.out[int64_t(b) * a.T + acc] = token;
    if (parts > 1) {  // the others' shared memory is read until here
        cluster_arrive_release();
        cluster_wait_acquire();
    }
}

template <int DT>
static cudaError_t launch_resample(const RaceArgs &a, int32_t B, cudaStream_t s) {
    int dev = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    const int parts = parts_of(B, (int64_t(a.V) + LogitRow<DT>::P - 1) / LogitRow<DT>::P, kRaceThreads, 2 * sms);
    return launch_pdl(resample_kernel<DT>, dim3(unsigned(parts), unsigned(B)), dim3(kRaceThreads), 0, s, parts > 1 ? unsigned(parts) : 0u, a, parts);
}

}  // namespace switchsd

using namespace switchsd;

extern "C" int switchsd_resample(const switchsd_resample_params *p) {
    if (!p || !p->logits || !p->draft_len || !p->seeds || !p->ctx_lens || !p->out) return SWITCHSD_ERR_ARG;
    if (p->dtype != SWITCHSD_BF16 && p->dtype != SWITCHSD_F16 && p->dtype != SWITCHSD_F32) return SWITCHSD_ERR_ARG;
    const uintptr_t size = p->dtype == SWITCHSD_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(p->logits) % size || reinterpret_cast<uintptr_t>(p->q_logits) % size) return SWITCHSD_ERR_ARG;
    if (p->T > 1 && (!p->draft || !p->p_draft || !p->u)) return SWITCHSD_ERR_ARG;
    if (p->T > 1 && p->q_logits && (!p->q_lse || !p->lse)) return SWITCHSD_ERR_ARG;
    if ((p->stride_b < 0 && p->B > 1) || (p->stride_t < 0 && p->T > 1)) return SWITCHSD_ERR_ARG;
    if (p->q_logits && ((p->q_stride_b < 0 && p->B > 1) || (p->q_stride_t < 0 && p->T > 2))) return SWITCHSD_ERR_ARG;
    if (p->B < 1 || p->B > 65535 || p->T < 1 || p->T > 262140 || p->V < 1 || p->V > SWITCHSD_VMAX) return SWITCHSD_ERR_SHAPE;
    RaceArgs a;
    a.logits = p->logits;
    a.q_logits = p->T > 1 ? p->q_logits : nullptr;
    a.sb = stride_of(p->stride_b, p->B);
    a.st = stride_of(p->stride_t, p->T);
    a.qb = stride_of(p->q_stride_b, p->B);
    a.qt = stride_of(p->q_stride_t, p->T - 1);
    a.lse = p->lse;
    a.q_lse = p->q_lse;
    a.temperature = p->temperature;
    a.p = p->p_draft;
    a.q = p->q_draft;
    a.u = p->u;
    a.draft = p->draft;
    a.draft_len = p->draft_len;
    a.mode = p->mode;
    a.ctx_lens = p->ctx_lens;
    a.seeds = p->seeds;
    a.out = p->out;
    a.status = p->status;
    a.T = p->T;
    a.V = p->V;
    cudaStream_t s = static_cast<cudaStream_t>(p->stream);
    const cudaError_t e = p->dtype == SWITCHSD_F32   ? launch_resample<SWITCHSD_F32>(a, p->B, s)
                          : p->dtype == SWITCHSD_F16 ? launch_resample<SWITCHSD_F16>(a, p->B, s)
                                                     : launch_resample<SWITCHSD_BF16>(a, p->B, s);
    return e == cudaSuccess ? SWITCHSD_OK : SWITCHSD_ERR_CUDA;
}
