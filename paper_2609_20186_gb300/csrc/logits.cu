// logits.cu -- switchsd_logits: penalties for repeated tokens, biases and grammar masks on the logits of B rows and T
// positions, and every position's greedy token.
//
// Two kernels.  The first counts: CTA (part, row) reads the row's context and counts its part of the vocabulary in shared
// memory (one word a token: output occurrences, and flags).  A token that is seen, biased or in the draft is special: a
// bit in the part's map, and an entry of its list, go to the workspace.  Chunks of 256 tokens go round the parts, because a
// tokenizer's low ids are the frequent ones.  The second streams: CTA (part, positions, row) reads its part of a few
// positions once, where everything but the specials meets the mask and a maximum; then goes through the part's list, 32
// lanes on 32 specials however they lie, each over those positions (the cache still has what is read again).  The parts'
// best tokens meet in a word of the workspace a position, and the last CTA of a group of positions writes the tokens.
//
// Each value is worked out in binary32, one rounding an operation, in the header's order, and the best is a maximum of
// (value, token), so nothing depends on the split or on who comes first.
//
// What bounds it: the instructions and latencies of both: the first looks at every token of the context once a part and
// adds up in shared memory, the second has 2 or 4 bytes an element to read (and write).  Measured: 64 rows of 8K to 32K
// tokens, 1 to 17 positions, 128,256 tokens, masks and biases: 89 us, 28 of them the counting (148 MB of logits are 22 us);
// 16 rows of 32K to 128K, 1 to 33 positions, 152,064 tokens, written: 108 us; one row and position: 12 us.  Measured and
// not kept: one kernel that counted and then streamed (126 us where the two took 104); the context cut over a cluster of
// the parts, with remote additions (118 us where each part reading it whole takes 94); sending for the first logits while
// the tokens are counted (no change).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "kv4.cuh"

namespace switchsd {

constexpr int kCountThreads = 512;
constexpr int kCountFlight = 4;             // vectors of four tokens of a thread in flight
constexpr int kLogitThreads = 256;
constexpr int kLogitWarps = kLogitThreads / kWarp;
constexpr int kLogitGroup = 4;              // positions of a CTA
constexpr int kLogitFlight = 4;             // units (32 vectors of 16 bytes) of a warp in flight, over its positions
constexpr int kChunk = 256;                 // tokens that lie together in a part
constexpr uint32_t kSeen = 1u << 31;        // in a token's word: occurs in the context
constexpr uint32_t kInDraft = 1u << 30;     // occurs in the draft
constexpr uint32_t kBiased = 1u << 29;      // is named by the biases
constexpr uint32_t kCount = kBiased - 1;    // output occurrences in the context and in the draft so far

struct LogitArgs {
    const uint8_t *logits;
    uint8_t *out;
    int64_t sb, st, ob, ot;  // strides in elements
    const int32_t *ctx, *lens, *draft, *new_lens, *prompt, *bias_ids;
    const float *rep, *freq, *pres, *bias;
    const uint32_t *mask;
    int32_t *argmax, *status;
    int32_t T, V, cap, draft_stride, new_add, nbias, mask_words;
    int32_t slice;           // places for tokens of a part, a multiple of kChunk
    int32_t parts_log;       // log2 of the parts
    int32_t groups;          // of positions
    int32_t entries;         // places of a part's list
    uint32_t hash_mask;      // places of the bias table less one
    int32_t marks;           // whether there are specials at all: penalties or biases
    // workspace
    unsigned long long *best;  // [B][T]
    uint32_t *done;            // [B][groups]
    int32_t *count;            // [B][parts]: entries of the lists
    uint32_t *bits;            // [B][parts][slice / 32]
    uint2 *list;               // [B][parts][entries]: place and bias entry + 1 (16 bits each), word
};

// Which tokens a part has: token v is in chunk v / kChunk, chunk c in part c % parts.
struct Part {
    int32_t V, part, log;
    __device__ bool has(int32_t v) const { return ((uint32_t(v) / kChunk) & ((1u << log) - 1)) == uint32_t(part); }
    __device__ int place_of(int32_t v) const { return int(((uint32_t(v) / kChunk) >> log) * kChunk | (uint32_t(v) & (kChunk - 1))); }
    __device__ int find(int32_t v) const { return uint32_t(v) < uint32_t(V) && has(v) ? place_of(v) : -1; }  // -1: not here
    __device__ int32_t token_at(int l) const { return ((((l / kChunk) << log) + part) * kChunk) | (l & (kChunk - 1)); }
    // places in use: every one below it names a token, but for the vocabulary's last chunk
    __device__ int used() const {
        const int chunks = (V + kChunk - 1) / kChunk;
        return (chunks > part ? ((chunks - part - 1) >> log) + 1 : 0) * kChunk;
    }
};

// A row's positions, and whether its lengths are good.
__device__ __forceinline__ int row_positions(const LogitArgs &a, int b, int32_t &L, bool &ok) {
    const int64_t n = a.new_lens ? int64_t(__ldcg(a.new_lens + b)) + a.new_add : a.T;
    L = a.lens ? __ldcg(a.lens + b) : 0;
    ok = n >= 0 && n <= a.T && L >= 0 && L <= a.cap;
    return ok ? int(n) : 0;
}

// An element type: widening, narrowing, a vector whose elements without their bit become -inf (lut: for every byte of
// bits, the mask of four words of two 16-bit elements), and a vector's largest
// element (NaN if they all are).
template <int DT>
struct Elem;
template <>
struct Elem<SWITCHSD_BF16> {
    using type = uint16_t;
    __device__ static float get(uint16_t v) { return bf16_lo(v); }
    __device__ static uint16_t put(float f) { return __bfloat16_as_ushort(__float2bfloat16_rn(f)); }
    __device__ static uint4 keep(uint4 w, uint32_t open, const uint4 *lut) {
        const uint4 m = lut[open & 255u];
        constexpr uint32_t none = 0xff80ff80u;
        return make_uint4((w.x & m.x) | (none & ~m.x), (w.y & m.y) | (none & ~m.y), (w.z & m.z) | (none & ~m.z), (w.w & m.w) | (none & ~m.w));
    }
    __device__ static uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ static float largest(uint4 w) {
        const uint32_t m = max2(max2(w.x, w.y), max2(w.z, w.w));
        return fmaxf(bf16_lo(m), bf16_hi(m));
    }
};
template <>
struct Elem<SWITCHSD_F16> {
    using type = uint16_t;
    __device__ static float get(uint16_t v) { return __half2float(__ushort_as_half(v)); }
    __device__ static uint16_t put(float f) { return __half_as_ushort(__float2half_rn(f)); }
    __device__ static uint4 keep(uint4 w, uint32_t open, const uint4 *lut) {
        const uint4 m = lut[open & 255u];
        constexpr uint32_t none = 0xfc00fc00u;
        return make_uint4((w.x & m.x) | (none & ~m.x), (w.y & m.y) | (none & ~m.y), (w.z & m.z) | (none & ~m.z), (w.w & m.w) | (none & ~m.w));
    }
    __device__ static uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t r;
        asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ static float largest(uint4 w) {
        const uint32_t m = max2(max2(w.x, w.y), max2(w.z, w.w));
        return fmaxf(get(uint16_t(m)), get(uint16_t(m >> 16)));
    }
};
template <>
struct Elem<SWITCHSD_F32> {
    using type = float;
    __device__ static float get(float v) { return v; }
    __device__ static float put(float f) { return f; }
    __device__ static uint4 keep(uint4 w, uint32_t open, const uint4 *) {
        constexpr uint32_t none = 0xff800000u;
        return make_uint4(open & 1 ? w.x : none, open & 2 ? w.y : none, open & 4 ? w.z : none, open & 8 ? w.w : none);
    }
    __device__ static float largest(uint4 w) {
        return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
    }
};

// A value's place in the order of values; -0 and 0 share one.  That of -inf is kNothing.
__device__ __forceinline__ uint32_t order_of(float v) {
    const uint32_t u = __float_as_uint(v + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
constexpr uint32_t kNothing = 0x007fffffu;
// (value, token) as a word whose order is larger value first, then smaller token; 0 is nothing.
__device__ __forceinline__ uint64_t best_key(uint32_t order, uint32_t id) { return (uint64_t(order) << 32) | uint32_t(~id); }

__device__ __forceinline__ uint32_t bias_hash(uint32_t id) { return (id * 0x9E3779B1u) >> 15; }

// Shared memory of the counting kernel, in words.
static size_t count_words(int32_t slice, uint32_t hash_places) { return size_t(slice) + size_t(slice) / 32 + 2 * size_t(hash_places); }

__global__ void __launch_bounds__(kCountThreads, 3) logits_count_kernel(const LogitArgs a) {
    extern __shared__ __align__(16) uint32_t smem[];
    __shared__ int32_t s_warp[kCountThreads / kWarp];
    const uint32_t places = a.nbias ? a.hash_mask + 1 : 0;
    uint32_t *cnt = smem, *bits = cnt + a.slice;                       // [slice], [slice / 32]
    int32_t *keys = reinterpret_cast<int32_t *>(bits + a.slice / 32);  // [places]: biased tokens, -1
    int32_t *vals = keys + places;                                     // [places]: last entry + 1
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.y, parts = int(gridDim.x);
    const Part part{a.V, int(blockIdx.x), a.parts_log};
    // everything here but the inputs: before the kernel ahead has finished
    const int words = a.slice / 32;
    for (int i = tid; i < a.slice / 4; i += kCountThreads) reinterpret_cast<uint4 *>(cnt)[i] = make_uint4(0, 0, 0, 0);
    for (int i = tid; i < int(places); i += kCountThreads) {
        keys[i] = -1;
        vals[i] = 0;
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    // What a row needs to know is read together, and its first tokens with it (the places are the row's, filled or not).
    int32_t L;
    bool ok;
    const int nw = row_positions(a, b, L, ok);
    const float rep = a.rep ? __ldcg(a.rep + b) : 1.f, freq = a.freq ? __ldcg(a.freq + b) : 0.f, pres = a.pres ? __ldcg(a.pres + b) : 0.f;
    const int32_t first = a.prompt ? __ldcg(a.prompt + b) : 0;
    const int32_t *ctx = a.ctx + size_t(b) * size_t(a.cap);
    auto fetch = [&](int i, int end) { return i < end ? __ldcg(reinterpret_cast<const int4 *>(ctx + i)) : make_int4(-1, -1, -1, -1); };
    int4 next[kCountFlight];
#pragma unroll
    for (int k = 0; k < kCountFlight; ++k) next[k] = fetch(4 * (tid + k * kCountThreads), a.marks ? a.cap : 0);
    int32_t draft = a.draft && tid < a.T - 1 ? __ldcg(a.draft + size_t(b) * a.draft_stride + tid) : -1;
    int32_t biased = tid < a.nbias ? __ldcg(a.bias_ids + size_t(b) * a.nbias + tid) : -1;
    if (part.part == 0) {
        if (tid == 0 && a.status) a.status[b] = ok ? SWITCHSD_ROW_OK : SWITCHSD_ROW_BAD_LEN;
        for (int t = tid; t < a.T; t += kCountThreads) {
            a.best[size_t(b) * a.T + t] = 0;
            if (t >= nw && a.argmax) a.argmax[size_t(b) * a.T + t] = -1;
        }
        for (int g = tid; g < a.groups; g += kCountThreads) a.done[size_t(b) * a.groups + g] = 0;
    }
    if (!a.marks || nw == 0) return;
    if (rep != 1.f || freq != 0.f || pres != 0.f) {
        for (int i0 = 4 * tid; i0 < L; i0 += 4 * kCountThreads * kCountFlight) {
#pragma unroll
            for (int k = 0; k < kCountFlight; ++k) {
                const int i = i0 + 4 * k * kCountThreads;
                if (i >= L) break;
                const int32_t id[4] = {next[k].x, next[k].y, next[k].z, next[k].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (!part.has(id[e])) continue;
                    const int at = part.place_of(id[e]);
                    if (uint32_t(id[e]) < uint32_t(a.V) && i + e < L) {
                        if (i + e < first)
                            atomicOr(&cnt[at], kSeen);
                        else
                            atomicAdd(&cnt[at], 1u);
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < kCountFlight; ++k) next[k] = fetch(i0 + 4 * kCountThreads * (kCountFlight + k), L);
        }
        if (a.draft)
            for (int i = tid; i < nw - 1; i += kCountThreads) {
                if (i != tid) draft = __ldcg(a.draft + size_t(b) * a.draft_stride + i);
                const int at = part.find(draft);
                if (at >= 0) atomicOr(&cnt[at], kInDraft);
            }
    }
    for (int i = tid; i < a.nbias; i += kCountThreads) {
        if (i != tid) biased = __ldcg(a.bias_ids + size_t(b) * a.nbias + i);
        const int at = part.find(biased);
        if (at < 0) continue;
        // at most half of the places are taken, so the search ends; the last entry that names the token stays
        for (uint32_t p = bias_hash(uint32_t(biased)) & a.hash_mask;; p = (p + 1) & a.hash_mask) {
            const int32_t was = atomicCAS(&keys[p], -1, biased);
            if (was == -1 || was == biased) {
                atomicMax(&vals[p], i + 1);
                break;
            }
        }
        atomicOr(&cnt[at], kBiased);
    }
    __syncthreads();
    uint32_t *out_bits = a.bits + (size_t(b) * parts + part.part) * words;
    for (int i = warp; i < words; i += kCountThreads / kWarp) {
        const uint32_t m = __ballot_sync(kFull, cnt[32 * i + lane] != 0);
        if (lane == 0) bits[i] = m;
    }
    __syncthreads();
    // The map goes out.  A warp lists the specials of words [warp per, + per), a lane those of a word, all in the order of
    // their places, so that neighbours in the list are near each other in the logits.
    const int per = (words + kCountThreads / kWarp - 1) / (kCountThreads / kWarp);
    const int w0 = min(words, warp * per), w1 = min(words, w0 + per);
    int mine = 0;
    for (int i = w0 + lane; i < w1; i += kWarp) {
        out_bits[i] = bits[i];
        mine += __popc(bits[i]);
    }
    mine = __reduce_add_sync(kFull, mine);
    if (lane == 0) s_warp[warp] = mine;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kCountThreads / kWarp; ++w) {
        if (w < warp) before += s_warp[w];
        all += s_warp[w];
    }
    if (tid == 0) a.count[size_t(b) * parts + part.part] = all;
    uint2 *list = a.list + (size_t(b) * parts + part.part) * a.entries;
    for (int i0 = w0; i0 < w1; i0 += kWarp) {
        const int i = i0 + lane;
        uint32_t m = i < w1 ? bits[i] : 0u;
        const int n = __popc(m);
        int k = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(kFull, k, o);
            if (lane >= o) k += y;
        }
        const int sum = __shfl_sync(kFull, k, 31);
        for (k += before - n; m; m &= m - 1, ++k) {
            const int at = 32 * i + __ffs(int(m)) - 1;
            const uint32_t w = cnt[at];
            uint32_t bias = 0;
            if (w & kBiased) {
                const int32_t v = part.token_at(at);
                uint32_t p = bias_hash(uint32_t(v)) & a.hash_mask;
                while (keys[p] != v) p = (p + 1) & a.hash_mask;
                bias = uint32_t(vals[p]);
            }
            if (k < a.entries) list[k] = make_uint2(uint32_t(at) | (bias << 16), w);
        }
        before += sum;
    }
}

// The positions of a CTA that the streaming pass takes together, P of them (the last ones may not be there), and what they
// have in common: rows begin at `row`, results at `out`, masks at `mask`, each its own stride apart.
template <int DT, int P>
__device__ __forceinline__ void stream_part(const LogitArgs &a, const Part &part, int positions, const typename Elem<DT>::type *row,
                                            typename Elem<DT>::type *out, const uint32_t *mask, const uint32_t *bits, const uint4 *lut,
                                            unsigned long long *s_best) {
    using E = Elem<DT>;
    using elem = typename E::type;
    constexpr int N = 16 / int(sizeof(elem));     // elements of a vector
    constexpr int kUnit = kWarp * N;              // tokens of a unit
    constexpr int kUnits = kLogitFlight / P;      // units of a warp in flight
    constexpr uint32_t kExact = 1u << 31;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int units = part.used() / kUnit;
    // The units that are read (and written) by vectors: all but the vocabulary's last tokens, where every row begins on a
    // 16-byte boundary; the rest 32 neighbours at a time.
    int whole = units;
    while (whole > 0 && part.token_at((whole - 1) * kUnit) + kUnit > a.V) --whole;
    {
        uintptr_t low = reinterpret_cast<uintptr_t>(row) | reinterpret_cast<uintptr_t>(out);
        if (positions > 1) low |= (uintptr_t(a.st) | (out ? uintptr_t(a.ot) : 0)) * sizeof(elem);
        if (low & 15) whole = 0;
    }
    // Per position, a lane's best value, and its token (kExact) or the first token of the vector that has it.
    float best[P];
    uint32_t where[P];
#pragma unroll
    for (int t = 0; t < P; ++t) {
        best[t] = -INFINITY;
        where[t] = 0;
    }
    const int step = (kLogitWarps * kUnit) << part.log;  // tokens between a warp's units: whole chunks
    auto open_of = [&](int t, int32_t v) { return uint32_t(__ldcg(reinterpret_cast<const uint8_t *>(mask + size_t(t) * a.mask_words) + (v >> 3))) >> (v & 7 & -N); };
    auto special_of = [&](int l) { return uint32_t(__ldcg(reinterpret_cast<const uint8_t *>(bits) + (l >> 3))) >> (l & 7 & -N); };
    for (int u0 = warp; u0 < whole; u0 += kUnits * kLogitWarps) {
        const int32_t v0 = part.token_at(u0 * kUnit) + lane * N;
        uint4 w[kUnits][P];
        uint32_t open[kUnits][P], special[kUnits];
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const bool in = u0 + i * kLogitWarps < whole;
            special[i] = a.marks && in ? special_of((u0 + i * kLogitWarps) * kUnit + lane * N) : 0u;
#pragma unroll
            for (int t = 0; t < P; ++t) {
                const int32_t v = v0 + i * step;
                open[i][t] = 0;
                w[i][t] = make_uint4(0, 0, 0, 0);
                if (in && t < positions) {
                    w[i][t] = *reinterpret_cast<const uint4 *>(row + t * a.st + v);
                    open[i][t] = mask ? open_of(t, v) : 0xffu;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kUnits; ++i)
#pragma unroll
            for (int t = 0; t < P; ++t) {
                const int32_t v = v0 + i * step;
                if (out && u0 + i * kLogitWarps < whole && t < positions)
                    *reinterpret_cast<uint4 *>(out + t * a.ot + v) = mask ? E::keep(w[i][t], open[i][t], lut) : w[i][t];
                const float m = E::largest(E::keep(w[i][t], open[i][t] & ~special[i], lut));
                if (m > best[t]) {  // a lane's tokens come in order, so only a larger value is better
                    best[t] = m;
                    where[t] = uint32_t(v);
                }
            }
    }
    for (int u = whole + (warp - whole % kLogitWarps + kLogitWarps) % kLogitWarps; u < units; u += kLogitWarps) {
        const int32_t v0 = part.token_at(u * kUnit);
        uint32_t special[N];
#pragma unroll
        for (int j = 0; j < N; ++j) special[j] = a.marks ? __ldcg(bits + u * (kUnit / 32) + j) : 0u;
#pragma unroll
        for (int t = 0; t < P; ++t) {
            if (t >= positions) break;
            elem y[N];
            uint32_t open[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int32_t v = v0 + 32 * j + lane;
                y[j] = v < a.V ? row[t * a.st + v] : elem(0);
                open[j] = v0 + 32 * j >= a.V ? 0u : mask ? __ldcg(mask + size_t(t) * a.mask_words + (v0 >> 5) + j) : 0xffffffffu;
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int32_t v = v0 + 32 * j + lane;
                const bool in = v < a.V, may = (open[j] >> lane) & 1;
                const float x = in && may && !((special[j] >> lane) & 1) ? E::get(y[j]) : -INFINITY;
                if (x > best[t]) {
                    best[t] = x;
                    where[t] = uint32_t(v) | kExact;
                }
                if (out && in) out[t * a.ot + v] = may ? y[j] : E::put(-INFINITY);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < P; ++t) {
        const uint32_t mine = order_of(best[t]), all = __reduce_max_sync(kFull, mine);
        if (all <= kNothing) continue;
        uint32_t id = 0xffffffffu;
        if (mine == all) {
            id = where[t] & ~kExact;
            if (!(where[t] & kExact)) {  // which of the vector: it is read again
                const int32_t v = int32_t(where[t]);
                const uint32_t may = (mask ? open_of(t, v) : 0xffu) & ~(a.marks ? special_of(part.place_of(v)) : 0u);
                elem y[N];
                *reinterpret_cast<uint4 *>(y) = *reinterpret_cast<const uint4 *>(row + t * a.st + v);
#pragma unroll
                for (int j = N - 1; j >= 0; --j)
                    if (((may >> j) & 1) && E::get(y[j]) == best[t]) id = uint32_t(v + j);
            }
        }
        id = __reduce_min_sync(kFull, id);
        if (lane == 0) atomicMax(&s_best[t], static_cast<unsigned long long>(best_key(all, id)));
    }
}

template <int DT>
__global__ void __launch_bounds__(kLogitThreads, 4) logits_kernel(const LogitArgs a) {
    using E = Elem<DT>;
    using elem = typename E::type;
    __shared__ unsigned long long s_best[kLogitGroup];
    __shared__ uint4 s_lut[DT == SWITCHSD_F32 ? 1 : 256];
    __shared__ int s_last;
    const int tid = threadIdx.x;
    const int b = blockIdx.z, t0 = int(blockIdx.y) * kLogitGroup, parts = int(gridDim.x);
    const Part part{a.V, int(blockIdx.x), a.parts_log};
    if (tid < kLogitGroup) s_best[tid] = 0;
    if (DT != SWITCHSD_F32 && tid < 256) {
        auto pair = [&](int i) { return ((tid >> i) & 1 ? 0xffffu : 0u) | ((tid >> (i + 1)) & 1 ? 0xffff0000u : 0u); };
        s_lut[tid] = make_uint4(pair(0), pair(2), pair(4), pair(6));
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    int32_t L;
    bool ok;
    const int t1 = min(t0 + kLogitGroup, row_positions(a, b, L, ok));
    if (t0 >= t1) return;
    const elem *rows = reinterpret_cast<const elem *>(a.logits) + int64_t(b) * a.sb;
    elem *outs = a.out ? reinterpret_cast<elem *>(a.out) + int64_t(b) * a.ob : nullptr;
    const uint32_t *masks = a.mask ? a.mask + size_t(b) * a.T * a.mask_words : nullptr;
    {
        const uint32_t *bits = a.bits + (size_t(b) * parts + part.part) * (a.slice / 32);
        const elem *row = rows + t0 * a.st;
        elem *out = outs ? outs + t0 * a.ot : nullptr;
        const uint32_t *mask = masks ? masks + size_t(t0) * a.mask_words : nullptr;
        if (t1 - t0 > 2)
            stream_part<DT, 4>(a, part, t1 - t0, row, out, mask, bits, s_lut, s_best);
        else if (t1 - t0 == 2)
            stream_part<DT, 2>(a, part, 2, row, out, mask, bits, s_lut, s_best);
        else
            stream_part<DT, 1>(a, part, 1, row, out, mask, bits, s_lut, s_best);
    }
    if (a.marks) {
        if (outs) __syncthreads();  // the specials' results go over what the vectors wrote in their places
        const float rep = a.rep ? __ldcg(a.rep + b) : 1.f, freq = a.freq ? __ldcg(a.freq + b) : 0.f, pres = a.pres ? __ldcg(a.pres + b) : 0.f;
        const int specials = min(__ldcg(a.count + size_t(b) * parts + part.part), a.entries);
        const uint2 *list = a.list + (size_t(b) * parts + part.part) * a.entries;
        const int32_t *draft = a.draft + size_t(b) * a.draft_stride;
        uint64_t top[kLogitGroup] = {};
        uint2 next = tid < specials ? __ldcg(list + tid) : make_uint2(0, 0);
        for (int s = tid; s < specials; s += kLogitThreads) {
            const uint2 entry = next;
            if (s + kLogitThreads < specials) next = __ldcg(list + s + kLogitThreads);
            const uint32_t w = entry.y;
            const int32_t v = part.token_at(int(entry.x & 0xffffu));
            const elem *p = rows + int64_t(t0) * a.st + v;
            bool may[kLogitGroup];
#pragma unroll
            for (int i = 0; i < kLogitGroup; ++i)
                may[i] = t0 + i < t1 && (!masks || ((__ldcg(masks + size_t(t0 + i) * a.mask_words + (v >> 5)) >> (v & 31)) & 1));
            float x[kLogitGroup];
#pragma unroll
            for (int i = 0; i < kLogitGroup; ++i) x[i] = may[i] ? E::get(p[i * a.st]) : 0.f;
            const float bias = w & kBiased ? __ldcg(a.bias + size_t(b) * a.nbias + (entry.x >> 16) - 1) : 0.f;
            uint32_t m = w & kCount;
            if (w & kInDraft)  // the draft's tokens behind the group's first position
                for (int d = 0; d < t0; ++d) m += __ldcg(draft + d) == v;
#pragma unroll
            for (int i = 0; i < kLogitGroup; ++i) {
                if (may[i]) {  // (what the mask leaves out has its -inf from the vectors)
                    float y = x[i];
                    if ((w & kSeen) || m) y = y > 0.f ? __fdiv_rn(y, rep) : __fmul_rn(y, rep);
                    if (m) y = __fsub_rn(__fsub_rn(y, __fmul_rn(freq, float(m))), pres);
                    if (w & kBiased) y = __fadd_rn(y, bias);
                    if (y > -INFINITY) top[i] = max(top[i], best_key(order_of(y), uint32_t(v)));
                    if (outs) outs[int64_t(t0 + i) * a.ot + v] = E::put(y);
                }
                if ((w & kInDraft) && t0 + i + 1 < t1) m += __ldcg(draft + t0 + i) == v;
            }
        }
#pragma unroll
        for (int i = 0; i < kLogitGroup; ++i) {
            const uint32_t high = __reduce_max_sync(kFull, uint32_t(top[i] >> 32));
            const uint32_t low = __reduce_max_sync(kFull, uint32_t(top[i] >> 32) == high ? uint32_t(top[i]) : 0u);
            if ((tid & 31) == 0 && high) atomicMax(&s_best[i], static_cast<unsigned long long>((uint64_t(high) << 32) | low));
        }
    }
    if (!a.argmax) return;
    __syncthreads();
    // the parts' best; the last part of these positions writes the tokens
    if (tid < t1 - t0) {
        if (s_best[tid]) atomicMax(&a.best[size_t(b) * a.T + t0 + tid], s_best[tid]);
        __threadfence();
    }
    __syncthreads();
    if (tid == 0) s_last = atomicAdd(&a.done[size_t(b) * a.groups + blockIdx.y], 1u) == uint32_t(parts - 1);
    __syncthreads();
    if (s_last && tid < t1 - t0) {
        __threadfence();
        const uint64_t key = __ldcg(&a.best[size_t(b) * a.T + t0 + tid]);
        a.argmax[size_t(b) * a.T + t0 + tid] = key ? int32_t(~uint32_t(key)) : -1;
    }
}

// log2 of the parts: enough that the shared memory of a part of the vocabulary leaves an SM two counting CTAs, and, where
// rows are few, more, up to about a CTA an SM -- as long as each part has a chunk.  Measured with and without the latter, in a
// graph: one row and position 12 and 16 us (with 64K tokens of context 25 and 34 us), 4 rows of 1 to 17 positions, masks and
// biases 26 and 31 us.
constexpr int kFewCtas = 128;
static int parts_log_of(int32_t V, int32_t B) {
    int log = V > 131072 ? 4 : V > 8192 ? 3 : 2;
    while ((int64_t(B) << (log + 1)) <= kFewCtas && (kChunk << (log + 1)) <= V) ++log;
    return log;
}
static int32_t slice_of(int32_t V, int log) { return (((V + kChunk - 1) / kChunk + (1 << log) - 1) >> log) * kChunk; }

// The workspace: sizes of its arrays, and their places after `base`.
static size_t logits_layout(const switchsd_logits_params *p, LogitArgs *a) {
    const int log = parts_log_of(p->V, p->B);
    const size_t B = size_t(p->B), parts = size_t(1) << log, slice = size_t(slice_of(p->V, log));
    const size_t groups = (size_t(p->T) + kLogitGroup - 1) / kLogitGroup;
    const bool marks = p->rep || p->freq || p->pres || p->nbias;
    // a part has no more specials than tokens, nor than the context, the draft and the biases name
    const size_t named = (p->ctx_tokens ? size_t(p->cap) : 0) + (p->draft ? size_t(p->T) : 0) + size_t(p->nbias);
    const size_t entries = marks ? std::min(slice, named) : 0;
    uint8_t *at = nullptr;
    if (a) {
        a->parts_log = log;
        a->slice = int32_t(slice);
        a->groups = int32_t(groups);
        a->entries = int32_t(entries);
        a->marks = marks && entries > 0;
        at = static_cast<uint8_t *>(p->workspace);
    }
    size_t size = 0;
    auto take = [&](size_t bytes) {
        uint8_t *q = at + size;
        size += (bytes + 15) / 16 * 16;
        return q;
    };
    uint8_t *best = take(B * size_t(p->T) * 8), *done = take(B * groups * 4), *count = take(B * parts * 4);
    uint8_t *bits = take(marks ? B * parts * (slice / 32) * 4 : 0), *list = take(B * parts * entries * 8);
    if (a) {
        a->best = reinterpret_cast<unsigned long long *>(best);
        a->done = reinterpret_cast<uint32_t *>(done);
        a->count = reinterpret_cast<int32_t *>(count);
        a->bits = reinterpret_cast<uint32_t *>(bits);
        a->list = reinterpret_cast<uint2 *>(list);
    }
    return size;
}

template <int DT>
static cudaError_t launch_logits(const LogitArgs &a, int B, cudaStream_t s) {
    static bool attr_done[64] = {false};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_done[dev]) {
        // the widest part and the largest bias table
        e = cudaFuncSetAttribute(logits_count_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(4 * count_words(16384, 2 * SWITCHSD_BIAS_MAX)));
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_done[dev] = true;
    }
    const unsigned parts = 1u << a.parts_log;
    // without specials the counting kernel only clears the positions' words
    const size_t smem = 4 * count_words(a.marks ? a.slice : 0, a.nbias ? a.hash_mask + 1 : 0);
    LogitArgs c = a;
    if (!a.marks) {
        c.slice = 0;
        c.nbias = 0;
    }
    e = launch_pdl(logits_count_kernel, dim3(a.marks ? parts : 1u, unsigned(B)), dim3(kCountThreads), smem, s, 0u, c);
    if (e != cudaSuccess) return e;
    return launch_pdl(logits_kernel<DT>, dim3(parts, unsigned(a.groups), unsigned(B)), dim3(kLogitThreads), 0, s, 0u, a);
}

}  // namespace switchsd

using namespace switchsd;

extern "C" size_t switchsd_logits_workspace_bytes(const switchsd_logits_params *p) {
    if (!p || p->B < 1 || p->T < 1 || p->V < 1 || p->V > SWITCHSD_VMAX || p->cap < 0 || p->nbias < 0) return 0;
    return logits_layout(p, nullptr);
}

extern "C" int switchsd_logits(const switchsd_logits_params *p) {
    if (!p || !p->logits || (!p->out && !p->argmax) || !p->workspace || !aligned16(p->workspace)) return SWITCHSD_ERR_ARG;
    if (p->dtype != SWITCHSD_BF16 && p->dtype != SWITCHSD_F16 && p->dtype != SWITCHSD_F32) return SWITCHSD_ERR_ARG;
    const uintptr_t size = p->dtype == SWITCHSD_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(p->logits) % size || reinterpret_cast<uintptr_t>(p->out) % size) return SWITCHSD_ERR_ARG;
    if ((p->ctx_tokens == nullptr) != (p->ctx_lens == nullptr) || (reinterpret_cast<uintptr_t>(p->ctx_tokens) & 15)) return SWITCHSD_ERR_ARG;
    if (p->nbias < 0 || (p->nbias > 0 && (!p->bias_ids || !p->bias))) return SWITCHSD_ERR_ARG;
    if (p->B < 1 || p->B > 65535 || p->T < 1 || p->V < 1 || p->V > SWITCHSD_VMAX || p->nbias > SWITCHSD_BIAS_MAX) return SWITCHSD_ERR_SHAPE;
    if (p->ctx_tokens && (p->cap < 4 || p->cap % 4 != 0 || p->cap >= (1 << 28))) return SWITCHSD_ERR_SHAPE;
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
    if (p->workspace_bytes < logits_layout(p, &a)) return SWITCHSD_ERR_ARG;
    if (a.groups > 65535) return SWITCHSD_ERR_SHAPE;
    a.hash_mask = 0;
    if (p->nbias) {
        uint32_t places = 2;
        while (places < 2u * uint32_t(p->nbias)) places *= 2;
        a.hash_mask = places - 1;
    }
    cudaStream_t s = static_cast<cudaStream_t>(p->stream);
    const cudaError_t e = p->dtype == SWITCHSD_F32    ? launch_logits<SWITCHSD_F32>(a, p->B, s)
                          : p->dtype == SWITCHSD_F16 ? launch_logits<SWITCHSD_F16>(a, p->B, s)
                                                     : launch_logits<SWITCHSD_BF16>(a, p->B, s);
    return e == cudaSuccess ? SWITCHSD_OK : SWITCHSD_ERR_CUDA;
}
