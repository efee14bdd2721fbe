// sampling.cuh -- rows of logits, as the operators that make probabilities and tokens of them read them.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv4.cuh"
#include "tc.cuh"

namespace switchsd {

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float log2_fast(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A row of V logits in vectors of 16 aligned bytes: vector j has the tokens j * P - lead .. j * P - lead + P - 1, of which
// the first and the last vector may lack some.
template <int DT>
struct LogitRow {
    using type = typename std::conditional<DT == SWITCHSD_F32, float, uint16_t>::type;
    static constexpr int P = 16 / int(sizeof(type));
    const type *row;
    int32_t V, lead, vectors;
    __device__ LogitRow(const void *base, int64_t at, int32_t v) : row(static_cast<const type *>(base) + at), V(v) {
        lead = int32_t((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(type));
        vectors = (V + lead + P - 1) / P;
    }
    __device__ static float widen(type v) {
        if constexpr (DT == SWITCHSD_F32)
            return v;
        else if constexpr (DT == SWITCHSD_F16)
            return __half2float(__ushort_as_half(v));
        else
            return bf16_lo(v);
    }
    __device__ float operator[](int32_t v) const {
        if constexpr (DT == SWITCHSD_F32)
            return __ldcg(row + v);
        else
            return widen(__ldcg(row + v));
    }
    __device__ int32_t token(int32_t j) const { return j * P - lead; }  // of vector j's first place (below 0: not there)
    __device__ static uint4 nothing() {
        constexpr uint32_t none = DT == SWITCHSD_F32 ? 0xff800000u : DT == SWITCHSD_F16 ? 0xfc00fc00u : 0xff80ff80u;
        return make_uint4(none, none, none, none);
    }
    // Places that the row does not have are -inf.
    __device__ __noinline__ static uint4 edge(const type *row, int32_t V, int32_t from) {
        uint32_t w[4];
        constexpr uint32_t none = DT == SWITCHSD_F32 ? 0xff800000u : DT == SWITCHSD_F16 ? 0xfc00u : 0xff80u;
        for (int e = 0; e < 4; ++e) {
            uint32_t x[4 / sizeof(type)];
            for (int i = 0; i < int(4 / sizeof(type)); ++i) {
                const int32_t v = from + e * int(4 / sizeof(type)) + i;
                x[i] = none;
                if (uint32_t(v) < uint32_t(V)) {
                    if constexpr (DT == SWITCHSD_F32)
                        x[i] = __float_as_uint(__ldcg(row + v));
                    else
                        x[i] = __ldcg(row + v);
                }
            }
            w[e] = DT == SWITCHSD_F32 ? x[0] : x[0] | (x[4 / sizeof(type) - 1] << 16);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ bool inside(int32_t j) const { return token(j) >= 0 && token(j) + P <= V; }
    __device__ bool all_inside(int32_t j, int32_t last, int32_t end) const { return token(j) >= 0 && last < end && token(last) + P <= V; }
    // Vectors j, j + step, ..; nothing from `end` on.  All loads are sent before the row's first or last vector is made up, for
    // which there is a call.
    template <int N>
    __device__ __forceinline__ void load(uint4 (&x)[N], int32_t j, int32_t step, int32_t end) const {
        if (all_inside(j, j + (N - 1) * step, end)) {
            const uint4 *from = reinterpret_cast<const uint4 *>(row + token(j));
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = __ldcs(from + i * step);
            return;
        }
        bool edges = false;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int32_t k = j + i * step;
            x[i] = nothing();
            if (k < end) {
                if (inside(k))
                    x[i] = __ldcs(reinterpret_cast<const uint4 *>(row + token(k)));
                else
                    edges = true;
            }
        }
        if (edges)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int32_t k = j + i * step;
                if (k < end && !inside(k)) x[i] = edge(row, V, token(k));
            }
    }
    // The same into shared memory, in flight until they are waited for: this thread's vectors, `width` apart.
    template <int N>
    __device__ __forceinline__ void fetch(uint4 *to, int32_t width, int32_t j, int32_t step, int32_t end) const {
        if (all_inside(j, j + (N - 1) * step, end)) {
            const uint4 *from = reinterpret_cast<const uint4 *>(row + token(j));
#pragma unroll
            for (int i = 0; i < N; ++i) cp_async16(to + i * width, from + i * step);
            return;
        }
        bool edges = false;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int32_t k = j + i * step;
            if (k < end && inside(k)) {
                cp_async16(to + i * width, row + token(k));
            } else {
                to[i * width] = nothing();
                edges |= k < end;
            }
        }
        if (edges)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int32_t k = j + i * step;
                if (k < end && !inside(k)) to[i * width] = edge(row, V, token(k));
            }
    }
    __device__ static void widen(uint4 w, float (&x)[P]) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (DT == SWITCHSD_F32) {
                x[e] = __uint_as_float(u[e]);
            } else if constexpr (DT == SWITCHSD_F16) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&u[e]));
                x[2 * e] = f.x;
                x[2 * e + 1] = f.y;
            } else {
                x[2 * e] = bf16_lo(u[e]);
                x[2 * e + 1] = bf16_hi(u[e]);
            }
        }
    }
    __device__ static uint32_t max2(uint32_t a, uint32_t b) {
        uint32_t r;
        if constexpr (DT == SWITCHSD_F16)
            asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        else
            asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    // A vector whose elements below kLow, and NaN, are kLow.
    static constexpr float kLow = DT == SWITCHSD_F16 ? -65504.f : -0x1.98p99f;  // (8 bits)
    __device__ static uint4 raised(uint4 w) {
        if constexpr (DT == SWITCHSD_F32) {
            return make_uint4(__float_as_uint(fmaxf(__uint_as_float(w.x), kLow)), __float_as_uint(fmaxf(__uint_as_float(w.y), kLow)),
                              __float_as_uint(fmaxf(__uint_as_float(w.z), kLow)), __float_as_uint(fmaxf(__uint_as_float(w.w), kLow)));
        } else {
            constexpr uint32_t low = DT == SWITCHSD_F16 ? 0xfbfffbffu : 0xf14cf14cu;
            return make_uint4(max2(w.x, low), max2(w.y, low), max2(w.z, low), max2(w.w, low));
        }
    }
    // The largest of N vectors' elements, NaN aside (NaN where there is nothing else).
    template <int N>
    __device__ static float largest(const uint4 (&w)[N]) {
        if constexpr (DT == SWITCHSD_F32) {
            float m = -INFINITY;
#pragma unroll
            for (int i = 0; i < N; ++i)
                m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(w[i].x), __uint_as_float(w[i].y)), fmaxf(__uint_as_float(w[i].z), __uint_as_float(w[i].w))));
            return m;
        } else {
            uint32_t m = max2(max2(w[0].x, w[0].y), max2(w[0].z, w[0].w));
#pragma unroll
            for (int i = 1; i < N; ++i) m = max2(m, max2(max2(w[i].x, w[i].y), max2(w[i].z, w[i].w)));
            return fmaxf(widen(type(m)), widen(type(m >> 16)));
        }
    }
};

// A value of type T in the shared memory of another CTA of the cluster.
__device__ __forceinline__ uint32_t remote_word(const void *p, uint32_t rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];\n" : "=r"(v) : "r"(map_to_rank(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ float remote_float(const void *p, uint32_t rank) { return __uint_as_float(remote_word(p, rank)); }

__device__ __forceinline__ void remote_store(void *p, uint32_t rank, int32_t x, int32_t y) {
    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};\n" ::"r"(map_to_rank(p, rank)), "r"(x), "r"(y) : "memory");
}

// CTAs of a row, a power of two: as many as leave every thread a vector, up to 8 (a cluster that every device takes), while
// the rows together stay within the CTAs that are on the GPU at once.
inline int parts_of(int64_t rows, int64_t vectors, int threads, int64_t resident) {
    int parts = 1;
    while (parts < 8 && rows * parts * 2 <= resident && vectors > int64_t(parts) * threads) parts *= 2;
    return parts;
}

}  // namespace switchsd
