// resample.cu -- switchsd_resample: the token that the sampled verification appends.
//
// An exponential race: with E_v exponential variables, the largest w_v / E_v is v with probability w_v / sum w, so one pass
// over the one row of logits that counts decides, without a sum over the vocabulary.  The random bits are a function of
// the row's seed, the token's place in the context and v.
//
// Screening.  E = -ln(1 - x) is at least x, so v beats a score s only where x < w_v e^-s: a binary exponential and a
// comparison of the number's upper 23 bits, beside the bits themselves (two 64-bit products for two tokens).  s is what a
// vector of logits a thread reaches at least; few tokens pass, and they alone are worked out, a thread each, in binary32.  Where two scores are closer than its error, both are worked out in binary64, so the answer is that of
// binary64 throughout.  A drafter's distribution is read for the few only: w = max(0, p - q) is at most p.
#include "sampling.cuh"

namespace switchsd {

constexpr int kRaceThreads = 512;
constexpr int kRaceFlight = 4;          // vectors of a thread in flight
constexpr int kRaceList = 1024;         // tokens of a CTA that passed the test
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
    // ln w - ln E of token v with logit z, -inf where it has no weight, or where it stays below `floor`.
    __device__ float score(int32_t v, float z, float floor) const {
        if (!(z > -INFINITY) || v == skip) return -INFINITY;
        if (greedy) return z;
        const uint32_t r = bits(v);
        const float e = r < 0x80000000u ? -log1pf(-(float(r) + 0.5f) * 0x1p-32f) : -logf((float(~r) + 0.5f) * 0x1p-32f);
        float y = z / temperature - logf(e);
        if (residual) {
            y -= lse;
            const float zq = q[v];
            if (zq > -INFINITY) {
                const float a = (zq - z) / temperature, b = q_lse - lse, d = a - b;  // ln(q / p), and how far it may be off
                const float off = 4e-7f * (fabsf(a) + fabsf(b));
                if (d > off) return -INFINITY;
                if (!(-d > 1e3f * off)) {  // p - q nearly cancels
                    if (y + logf(off - d) + margin(y) < floor) return -INFINITY;
                    return float(exact(v));
                }
                y += logf(-expm1f(d));
            }
        }
        return y;
    }
    // How far binary32's score may be off, and binary64's of what is compared with it.
    __device__ float margin(float s) const { return greedy || fabsf(s) == INFINITY ? 0.f : (residual ? 4e-3f : 2e-5f) + 1e-6f * fabsf(s); }
};

template <int DT>
struct Best {
    float s = -INFINITY;
    int32_t v = -1;
    __device__ void consider(const Race<DT> &race, int32_t token, float z, float floor) {
        const float x = race.score(token, z, floor);
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
    __shared__ int32_t s_first, s_best, s_n, s_few, s_token;
    __shared__ int32_t s_tokens[kRaceList];
    __shared__ int32_t s_list[kRaceThreads];
    __shared__ double s_exact[kRaceThreads];
    const int tid = threadIdx.x, part = blockIdx.x, b = blockIdx.y, k = a.T - 1;
    pdl_wait();
    pdl_trigger();
    // what does not depend on the accepted length is read together
    const int32_t len = __ldcg(a.draft_len + b), ctx = __ldcg(a.ctx_lens + b), mode = a.mode ? __ldcg(a.mode + b) : SWITCHSD_MODE_COPY + 1;
    const float temperature = a.temperature ? __ldcg(a.temperature + b) : 1.f;
    const uint64_t seed = uint64_t(__ldcg(a.seeds + b));
    auto rejected = [&](int i) {
        const int64_t at = int64_t(b) * k + i;
        const float q = a.q ? __ldcg(a.q + at) : 1.f;
        return !(__fmul_rn(__ldcg(a.u + at), q) < __ldcg(a.p + at));
    };
    const bool mine = tid < k && rejected(tid);
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
        s_n = s_few = 0;
        s_best = float_order(-INFINITY);
    }
    __syncthreads();
    if (mine && tid < len) atomicMin(&s_first, tid);
    for (int i = tid + kRaceThreads; i < len; i += kRaceThreads)
        if (rejected(i)) {
            atomicMin(&s_first, i);
            break;
        }
    __syncthreads();
    const int acc = s_first;
    if (part == 0)
        for (int i = tid; i < a.T; i += kRaceThreads)
            if (i != acc) a.out[int64_t(b) * a.T + i] = -1;
    // --- the weights ----------------------------------------------------------------------------------------------
    const bool drafted = acc < len, drafter = drafted && a.q_logits && mode != SWITCHSD_MODE_COPY;
    const Row row(a.logits, b * a.sb + acc * a.st, a.V);
    Race<DT> race{row, drafter ? Row(a.q_logits, b * a.qb + acc * a.qt, a.V) : row};
    race.key = splitmix(seed + (uint64_t(ctx) + uint64_t(acc) + 1) * kGolden);
    race.temperature = temperature;
    race.greedy = race.temperature == 0.f;
    race.residual = drafter && !race.greedy;
    race.lse = race.residual ? __ldcg(a.lse + int64_t(b) * a.T + acc) : 0.f;
    race.q_lse = race.residual ? __ldcg(a.q_lse + int64_t(b) * k + acc) : 0.f;
    race.skip = drafted && !drafter && !race.greedy ? __ldcg(a.draft + int64_t(b) * k + acc) : -1;
    const bool none = !(race.temperature >= 0.f && race.temperature < INFINITY) || race.lse != race.lse || race.q_lse != race.q_lse;
    const int32_t per = (row.vectors + parts - 1) / parts, begin = part * per, end = min(begin + per, row.vectors);
    const float c2 = fminf(kRaceLog2e / race.temperature, 3e38f);
    Best<DT> best;
    int32_t token = -1;
    bool again = race.residual || race.skip >= 0;  // where w leaves nothing
    while (!none) {
        if (race.greedy) {
            for (int32_t j = begin + tid; j < end; j += kRaceThreads) {
                uint4 w[1];
                float x[P];
                row.load(w, j, 0, end);
                Row::widen(w[0], x);
#pragma unroll
                for (int e = 0; e < P; ++e)
                    if (x[e] > best.s) {  // (ascending tokens)
                        best.s = x[e];
                        best.v = row.token(j) + e;
                    }
            }
        } else {
            uint4 w[F];
            row.load(w, begin + tid, kRaceThreads, end);
            // --- a bound: what a vector a thread reaches at least, in binary logarithms ---------------------------
            // E <= x (1 + x) for x <= 1/2, and ln(1 + x) <= x
            const float lse2 = race.lse * kRaceLog2e, q_lse2 = race.q_lse * kRaceLog2e;
            float low = -INFINITY;
            if (begin + tid < end && (!race.residual || (race.q.lead == race.l.lead && race.l.inside(begin + tid)))) {
                float x[P], y[P];
                Row::widen(w[0], x);
                if (race.residual) {
                    uint4 qw[1];
                    race.q.load(qw, begin + tid, 0, end);
                    Row::widen(qw[0], y);
                }
                const int32_t from = row.token(begin + tid);
                const float c = kRaceLog2e / race.temperature, eps = 1e-4f + 1e-6f * (fabsf(lse2) + fabsf(q_lse2));
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    const int32_t v = from + e;
                    const float r = (float(race.bits(v)) + 0.5f) * 0x1p-32f;
                    float z = fmaf(x[e], c, -lse2);
                    if (race.residual) {  // p - q less what their roundings may take
                        const float p = exp2_fast(z);
                        z = log2_fast(fmaf(-1.f - eps, exp2_fast(fmaf(y[e] > -INFINITY ? y[e] : -1e30f, c, -q_lse2)), (1.f - eps) * p));
                    }
                    z -= log2_fast(r) + 1.4427f * r;
                    if (uint32_t(v) < uint32_t(a.V) && v != race.skip && r <= 0.5f && x[e] > -INFINITY && fabsf(z) < 1e30f) low = fmaxf(low, z);
                }
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) low = fmaxf(low, __shfl_xor_sync(kFull, low, o));
            if ((tid & 31) == 0) atomicMax(&s_best, float_order(low));
            __syncthreads();
            low = order_float(s_best);
            // less what the roundings of the bound and of the test may take
            const float off = fabsf(low) < 1e30f ? 2e-3f + 1e-6f * (fabsf(low) + fabsf(lse2) + fabsf(q_lse2)) - low - lse2 : INFINITY;
            const float floor = fabsf(low) < 1e30f ? (low - 2e-3f - 1e-6f * (fabsf(low) + fabsf(lse2) + fabsf(q_lse2))) * 0.69314718f : -INFINITY;
            __syncthreads();
            if (tid == 0) s_best = float_order(-INFINITY);
            const uint64_t c22 = pair_of(c2, c2), off2 = pair_of(off, off), up = pair_of(1.002f, 1.002f), one = pair_of(1.0000003f, 1.0000003f);
            // --- the tokens that may be better --------------------------------------------------------------------
            uint4 next[F];
            for (int32_t base = begin + tid; base < end; base += kRaceThreads * F) {
                row.load(next, base + kRaceThreads * F, kRaceThreads, end);
                uint32_t mask = 0;
#pragma unroll
                for (int i = 0; i < F; ++i) {
                    float x[P], most[P];
                    Row::widen(w[i], x);
                    // 1 + (x rounded down to 23 bits) <= 1 + w e^-s
#pragma unroll
                    for (int e = 0; e < P; e += 2) {
                        const float2 z = halves_of(fma_pair(pair_of(x[e], x[e + 1]), c22, off2));
                        const float2 t = halves_of(fma_pair(pair_of(exp2_fast(z.x), exp2_fast(z.y)), up, one));
                        most[e] = t.x;
                        most[e + 1] = t.y;
                    }
                    const int32_t from = row.token(base + i * kRaceThreads);
                    uint64_t n = race.key + (uint64_t(int64_t(from >> 1)) + 1) * kGolden;  // of the pair that `from` lies in
                    auto test = [&](int e, uint32_t r) {
                        if (__uint_as_float(0x3f800000u | (r >> 9)) <= most[e]) mask |= 1u << (i * P + e);
                    };
                    if (row.lead & 1) {
                        uint64_t z = splitmix(n);
#pragma unroll
                        for (int e = 0; e < P; e += 2) {
                            test(e, uint32_t(z >> 32));
                            z = splitmix(n += kGolden);
                            test(e + 1, uint32_t(z));
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < P; e += 2, n += kGolden) {
                            const uint64_t z = splitmix(n);
                            test(e, uint32_t(z));
                            test(e + 1, uint32_t(z >> 32));
                        }
                    }
                }
                while (mask) {
                    const int at_mask = __ffs(int(mask)) - 1;
                    mask &= mask - 1;
                    const int32_t j = base + at_mask / P * kRaceThreads, v = row.token(j) + at_mask % P;
                    if (j >= end || uint32_t(v) >= uint32_t(a.V)) continue;
                    const int at = atomicAdd(&s_few, 1);
                    if (at < kRaceList)
                        s_tokens[at] = v;
                    else
                        best.consider(race, v, row[v], floor);
                }
#pragma unroll
                for (int i = 0; i < F; ++i) w[i] = next[i];
            }
            // --- their scores -------------------------------------------------------------------------------------
            __syncthreads();
            for (int i = tid; i < min(s_few, kRaceList); i += kRaceThreads) best.consider(race, s_tokens[i], row[s_tokens[i]], floor);
        }
        // --- the CTA's best: among those that binary32 does not tell from it, binary64's --------------------------
        float s = best.s;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s = fmaxf(s, __shfl_xor_sync(kFull, s, o));
        if ((tid & 31) == 0) atomicMax(&s_best, float_order(s));
        __syncthreads();
        const float top = order_float(s_best);
        if (top > -INFINITY && best.v >= 0 && best.s >= top - 2.f * race.margin(top)) s_list[atomicAdd(&s_n, 1)] = best.v;
        __syncthreads();
        const int n = s_n;
        if (n > 1) {
            if (tid < n) s_exact[tid] = race.exact(s_list[tid]);
            __syncthreads();
        }
        if (tid == 0) {
            int32_t v = n > 0 ? s_list[0] : -1;
            double most = n > 1 ? s_exact[0] : 0.;
            for (int i = 1; i < n; ++i)
                if (s_exact[i] > most || (s_exact[i] == most && s_list[i] < v)) {
                    v = s_list[i];
                    most = s_exact[i];
                }
            s_token = v;
        }
        // --- the row's --------------------------------------------------------------------------------------------
        if (parts > 1) {
            cluster_arrive_release();
            cluster_wait_acquire();
        }
        if (tid < 32 && (part == 0 || again)) {  // lane r has part r's
            int32_t v = -1;
            float its = -INFINITY;
            const int lane = tid;
            if (lane < parts) {
                v = parts > 1 ? int32_t(remote_word(&s_token, lane)) : s_token;
                its = parts > 1 ? order_float(int32_t(remote_word(&s_best, lane))) : top;
            }
            float all = its;
#pragma unroll
            for (int o = 4; o > 0; o >>= 1) all = fmaxf(all, __shfl_xor_sync(kFull, all, o));
            all = __shfl_sync(kFull, all, 0);
            uint32_t near = __ballot_sync(kFull, v >= 0 && its >= all - 2.f * race.margin(all));
            if (near & (near - 1)) {  // several: binary64's best, of equal ones the first
                double mine = -INFINITY;
                if ((near >> lane) & 1) mine = race.exact(v);
                int32_t best_v = -1;
                double most = -INFINITY;
                for (int r = 0; r < parts; ++r) {
                    const double x = __shfl_sync(kFull, mine, r);
                    const int32_t u = __shfl_sync(kFull, v, r);
                    if (((near >> r) & 1) && (best_v < 0 || x > most || (x == most && u < best_v))) {
                        best_v = u;
                        most = x;
                    }
                }
                token = best_v;
            } else if (near) {
                token = __shfl_sync(kFull, v, __ffs(int(near)) - 1);
            }
            if (lane == 0) s_first = token;  // (the accepted length is known)
        }
        if (!again) break;
        __syncthreads();
        if (s_first >= 0) break;
        // nothing is left of w: once more with p
        if (parts > 1) {
            cluster_arrive_release();  // (all have read the parts' results)
            cluster_wait_acquire();
        }
        if (tid == 0) {
            s_few = s_n = 0;
            s_best = float_order(-INFINITY);
        }
        __syncthreads();
        race.residual = again = false;
        race.lse = race.q_lse = 0.f;
        race.skip = -1;
    }
    if (part == 0 && tid == 0) a.out[int64_t(b) * a.T + acc] = token;
    if (parts > 1) {  // the parts' shared memory is read until here
        cluster_arrive_release();
        cluster_wait_acquire();
    }
}

template <int DT>
static cudaError_t launch_resample(const RaceArgs &a, int32_t B, cudaStream_t s) {
    const int sms = sm_count();
    if (sms == 0) return cudaErrorInvalidDevice;
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
