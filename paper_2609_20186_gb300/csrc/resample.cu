// resample.cu -- switchsd_resample: the token that the sampled verification appends.
//
// An exponential race: with E_v exponential variables, the largest w_v / E_v is v with probability w_v / sum w, so one pass
// over the one row of logits that counts decides, without a sum over the vocabulary.  The random bits are a function of
// the row's seed, the token's place in the context and v.
//
// Screening.  E = -ln(1 - x) is at least x, so v beats a score s only where x < w_v e^-s: a binary exponential and a
// comparison of the number's upper 23 bits, beside the bits themselves (two 64-bit products for two tokens).  s is what a
// vector of logits a thread reaches at least; few tokens pass (1 to 40 of a CTA), and they alone are worked out, a thread each,
// in binary32.  Where two scores are closer than its error, both are worked out in binary64, so the answer is that of binary64
// throughout.  A drafter's distribution is read for the few only: w = max(0, p - q) is at most p.
//
// Bound: latency, and the bits.  64 rows of 128,256 bf16 logits: 17 us, of which 2.3 pass until the accepted length is known, 2
// until the bound is, 6 in the screening (30 instructions a pair of tokens, most of them on the pipe of shifts and
// exclusive-ors) and 2 in the scores and the meeting; a launch takes the rest.  16 rows of 152,064, f16, with drafters'
// distributions: 16 us.  One CTA a row instead of a cluster: 26 and 49.  Testing the vector's largest logit with its smallest x instead of every
// token: 17.5 and 20, since several times as many are worked out; four vectors in flight instead of two: 17.1 and 17.3.
// Without a bound where a drafter's rows are aligned otherwise than the target's (odd vocabularies), 16 rows of 128,255: 95 us
// instead of 16.
#include "sampling.cuh"

namespace switchsd {

constexpr int kRaceThreads = 512;
constexpr int kRaceFlight = 2;          // vectors of a thread that are worked on, and as many in flight
constexpr int kRaceList = 1024;         // tokens of a CTA that passed the test
constexpr int kRaceWarps = kRaceThreads / kWarp, kRaceParts = 8;
constexpr float kRaceLog2e = 1.4426950408889634f;
constexpr float kRaceMost = 3.402823466e38f;  // binary32's largest

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
    // The bits of P tokens from `from` on, the first of a pair or (ODD) the second.
    template <bool ODD, int P>
    __device__ __forceinline__ void bits_of(int32_t from, uint32_t (&r)[P]) const {
        uint64_t n = key + (uint64_t(int64_t(from >> 1)) + 1) * kGolden, z = ODD ? splitmix(n) : 0;
#pragma unroll
        for (int e = 0; e < P; e += 2) {
            if (ODD) {
                r[e] = uint32_t(z >> 32);
                r[e + 1] = uint32_t(z = splitmix(n += kGolden));
            } else {
                z = splitmix(n);
                r[e] = uint32_t(z);
                r[e + 1] = uint32_t(z >> 32);
                n += kGolden;
            }
        }
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
        float y = fmaxf(z / temperature, -kRaceMost);  // (what binary32 does not reach has a weight, and binary64 tells it apart)
        if (residual) {
            y -= lse;  // ln p; a residual's p is binary64's, which has nothing below e^-745.14 and few bits from e^-708 on
            if (y + margin(y) < -745.2f) return -INFINITY;
            if (y - margin(y) < -700.f) return float(exact(v));
        }
        y -= logf(e);
        if (y + margin(y) < floor) return -INFINITY;  // (w is at most p)
        if (residual) {
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
    // How far binary32's score may be off, and binary64's of what is compared with it.  (A residual's is what is left of z /
    // temperature less lse: four roundings of 2^-24 of numbers up to |s| + |lse| and some 30 in size, twice.)
    __device__ float margin(float s) const {
        if (greedy || fabsf(s) == INFINITY) return 0.f;
        return residual ? 4e-3f + 1e-6f * (fabsf(s) + fabsf(lse)) : 2e-5f + 1e-6f * fabsf(s);
    }
};

template <int DT>
struct Best {
    float s = -INFINITY;
    int32_t v = -1;
    __device__ void consider(const Race<DT> &race, int32_t token, float x) {  // x: its score
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
    // The warp's: among those that binary32 does not tell from the best, binary64's best, of equal ones the first.
    __device__ void of_warp(const Race<DT> &race) {
        const int lane = threadIdx.x & 31;
        const float top = order_float(__reduce_max_sync(kFull, float_order(s)));
        const uint32_t near = __ballot_sync(kFull, v >= 0 && s >= top - 2.f * race.margin(top));
        int src = near ? __ffs(int(near)) - 1 : 0;
        if (near & (near - 1)) {
            double mine = -INFINITY, most = -INFINITY;
            if ((near >> lane) & 1) mine = race.exact(v);
            int32_t best_v = -1;
            for (uint32_t rest = near; rest; rest &= rest - 1) {
                const int r = __ffs(int(rest)) - 1;
                const double x = __shfl_sync(kFull, mine, r);
                const int32_t u = __shfl_sync(kFull, v, r);
                if (best_v < 0 || x > most || (x == most && u < best_v)) {
                    best_v = u;
                    most = x;
                    src = r;
                }
            }
        }
        s = __shfl_sync(kFull, s, src);
        v = __shfl_sync(kFull, v, src);
    }
};

template <int DT>
__global__ void __launch_bounds__(kRaceThreads, 2) resample_kernel(const RaceArgs a, int parts) {
    using Row = LogitRow<DT>;
    constexpr int P = Row::P, F = kRaceFlight;
    __shared__ int32_t s_few, s_token;
    __shared__ int32_t s_tokens[kRaceList];
    __shared__ float s_low[kRaceWarps];
    __shared__ __align__(8) int2 s_best[2][kRaceParts * kRaceWarps];  // by round: all warps' best scores and their tokens
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
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
    const bool mine = lane < k && rejected(lane);
    const bool ok = len >= 0 && len <= k && ctx >= 0;
    if (part == 0) {
        if (tid == 0 && a.status) a.status[b] = ok ? SWITCHSD_ROW_OK : SWITCHSD_ROW_BAD_LEN;
        if (!ok)
            for (int i = tid; i < a.T; i += kRaceThreads) a.out[int64_t(b) * a.T + i] = -1;
    }
    if (!ok) return;
    // --- the accepted length --------------------------------------------------------------------------------------
    uint32_t no = __ballot_sync(kFull, mine && lane < len);  // (every warp finds it for itself)
    int acc = no ? __ffs(int(no)) - 1 : len;
    for (int i = kWarp; no == 0 && i < len; i += kWarp) {
        no = __ballot_sync(kFull, i + lane < len && rejected(i + lane));
        if (no) acc = i + __ffs(int(no)) - 1;
    }
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
    int32_t token = -1;
    bool again = race.residual || race.skip >= 0;  // where w leaves nothing
    if (parts > 1 && !none) cluster_arrive_release();  // (that it runs: the others will write its shared memory)
    for (int round = 0; !none; ++round) {
        Best<DT> best;
        if (tid == 0) s_few = 0;
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
            const float lse2 = race.lse * kRaceLog2e, q_lse2 = race.q_lse * kRaceLog2e;
            float off, floor;
            auto look_at = [&](int32_t v) { best.consider(race, v, race.score(v, row[v], floor)); };
            auto screen = [&](auto odd) {  // (whether vectors begin with the second token of a pair is known to its loops)
                uint4 w[F], next[F];
                row.load(w, begin + tid, kRaceThreads, end);
                // --- a bound: what a vector a thread reaches at least, in binary logarithms -----------------------
                // E <= x (1 + x) for x <= 1/2, and ln(1 + x) <= x
                float low = -INFINITY;
                if (begin + tid < end && (!race.residual || race.l.inside(begin + tid))) {
                    float x[P], y[P];
                    Row::widen(w[0], x);
                    if (race.residual) {
                        uint4 qw[1];
                        if (race.q.lead == race.l.lead) {
                            race.q.load(qw, begin + tid, 0, end);
                            Row::widen(qw[0], y);
                        } else {  // (its vectors are other tokens')
#pragma unroll
                            for (int e = 0; e < P; ++e) y[e] = race.q[row.token(begin + tid) + e];
                        }
                    }
                    const int32_t from = row.token(begin + tid);
                    uint32_t bits[P];
                    race.template bits_of<odd, P>(from, bits);
                    const float c = kRaceLog2e / race.temperature, eps = 1e-4f + 1e-6f * (fabsf(lse2) + fabsf(q_lse2));
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        const int32_t v = from + e;
                        const float r = (float(bits[e]) + 0.5f) * 0x1p-32f;
                        float z = fmaf(x[e], c, -lse2);
                        if (race.residual) {  // p - q less what their roundings may take
                            const float p = exp2_fast(z);
                            z = log2_fast(fmaf(-1.f - eps, exp2_fast(fmaf(y[e] > -INFINITY ? y[e] : -1e30f, c, -q_lse2)), (1.f - eps) * p));
                        }
                        z -= log2_fast(r) + 1.4427f * r;
                        if (uint32_t(v) < uint32_t(a.V) && v != race.skip && r <= 0.5f && x[e] > -INFINITY && fabsf(z) < 1e30f) low = fmaxf(low, z);
                    }
                }
                low = order_float(__reduce_max_sync(kFull, float_order(low)));
                if (lane == 0) s_low[warp] = low;
                __syncthreads();
                low = order_float(__reduce_max_sync(kFull, float_order(s_low[lane % kRaceWarps])));
                // less what the roundings of the bound and of the test may take
                const float slack = 2e-3f + 1e-6f * (fabsf(low) + fabsf(lse2) + fabsf(q_lse2));
                off = fabsf(low) < 1e30f ? slack - low - lse2 : INFINITY;
                floor = fabsf(low) < 1e30f ? (low - slack) * 0.69314718f : -INFINITY;
                // --- the tokens that may be better ----------------------------------------------------------------
                for (int32_t base = begin + tid; base < end; base += kRaceThreads * F) {
                    row.load(next, base + kRaceThreads * F, kRaceThreads, end);
                    uint32_t mask = 0;
#pragma unroll
                    for (int i = 0; i < F; ++i) {
                        float x[P];
                        uint32_t r[P];
                        Row::widen(w[i], x);
                        // 1 + (x rounded down to 23 bits) <= 1 + w e^-s
                        race.template bits_of<odd, P>(row.token(base + i * kRaceThreads), r);
#pragma unroll
                        for (int e = 0; e < P; e += 2) {
                            const float2 z = halves_of(fma_pair(pair_of(x[e], x[e + 1]), pair_of(c2, c2), pair_of(off, off)));
                            const float2 t = halves_of(fma_pair(pair_of(exp2_fast(z.x), exp2_fast(z.y)), pair_of(1.002f, 1.002f), pair_of(1.0000003f, 1.0000003f)));
                            mask |= uint32_t(__uint_as_float(0x3f800000u | (r[e] >> 9)) <= t.x) << (i * P + e);
                            mask |= uint32_t(__uint_as_float(0x3f800000u | (r[e + 1] >> 9)) <= t.y) << (i * P + e + 1);
                        }
                    }
                    for (; mask; mask &= mask - 1) {
                        const int at_mask = __ffs(int(mask)) - 1;
                        const int32_t j = base + at_mask / P * kRaceThreads, v = row.token(j) + at_mask % P;
                        if (j >= end || uint32_t(v) >= uint32_t(a.V)) continue;
                        const int at = atomicAdd(&s_few, 1);
                        if (at < kRaceList)
                            s_tokens[at] = v;
                        else
                            look_at(v);
                    }
#pragma unroll
                    for (int i = 0; i < F; ++i) w[i] = next[i];
                }
            };
            if (row.lead & 1)
                screen(std::true_type{});
            else
                screen(std::false_type{});
            // --- their scores -------------------------------------------------------------------------------------
            __syncthreads();
            for (int i = tid; i < min(s_few, kRaceList); i += kRaceThreads) look_at(s_tokens[i]);
        }
        // --- the row's best, of all its warps' --------------------------------------------------------------------
        best.of_warp(race);
        if (parts > 1) {
            if (round == 0) cluster_wait_acquire();
            if (lane < parts) remote_store(&s_best[round][part * kRaceWarps + warp], uint32_t(lane), __float_as_int(best.s), best.v);
            cluster_arrive_release();
            cluster_wait_acquire();
        } else {
            if (lane == 0) s_best[round][warp] = make_int2(__float_as_int(best.s), best.v);
            __syncthreads();
        }
        if (warp == 0) {
            best = Best<DT>{};
            for (int i = lane; i < parts * kRaceWarps; i += kWarp)
                if (s_best[round][i].y >= 0) best.consider(race, s_best[round][i].y, __int_as_float(s_best[round][i].x));
            best.of_warp(race);
            token = best.v;
        }
        if (!again) break;
        if (tid == 0) s_token = token;
        __syncthreads();
        if (s_token >= 0) break;
        // nothing is left of w: once more with p
        race.residual = again = false;
        race.lse = race.q_lse = 0.f;
        race.skip = -1;
    }
    if (part == 0 && tid == 0) a.out[int64_t(b) * a.T + acc] = token;
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
