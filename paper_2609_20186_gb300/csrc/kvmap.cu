// kvmap.cu -- switchsd_kv_map: block tables and slot maps of a paged cache from the rows' device lengths.
//
// Two exclusive prefix sums over the rows decide everything: of the pages that rows give back (their places on the
// stack) and of the pages that rows ask for (their distance from its top).  A row either gives or asks, so both
// sums ride in one 64-bit scan.
//
// One cluster of CTAs, each with 32 rows of every 32 * CTAs in turn (a warp a row, more where rows are few); every CTA
// works out all rows' sums for itself, which costs less than handing them round, and cluster barriers stand between the
// gives, the takes and the slots.  As many CTAs as there are 32s of rows, 8 at most.  Measured, two calls of which a third
// of the rows begin or end (up to 512 pages each), one CTA against that rule: 128 rows 37 and 24 us, 1024 rows 171 and
// 45 us, 8192 rows 1147 and 214 us; a second CTA for 16 rows only waits (in a graph 14.2 us with one and 16.1 with two).
//
// What bounds it: latency -- the launch, and about four dependent trips to L2 (lengths, stack, table, slots); two calls
// on 64 rows take 13 us in a graph.  With many rows, the scattered 4-byte moves of pages, 128 of a row in flight.
#include "kv4.cuh"

namespace switchsd {

constexpr int kMapThreads = 1024;
constexpr int kMapWarps = kMapThreads / kWarp;
constexpr int kMapCtas = 8;  // of the cluster at most: the size that every device takes

struct MapArgs {
    const int32_t *lens, *new_lens;
    int32_t *table, *held, *free_list, *free_count, *slots, *status, *granted;
    int32_t B, T, blocks, pages, page_shift, lens_add, new_add;
};

// Exclusive scan over the CTA's threads of a pair of sums in one 64-bit word; `total` is the sum of all.
__device__ __forceinline__ uint64_t block_scan(uint64_t v, uint64_t *s_warp, uint64_t &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint64_t x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint64_t y = __shfl_up_sync(kFull, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();  // the last call's readers of s_warp are done
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    uint64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kMapWarps; ++w) {
        const uint64_t y = s_warp[w];
        if (w < warp) before += y;
        all += y;
    }
    total = all;
    return before + x - v;
}

// f(j, load(j)) for j = begin, begin + step, ..., with the loads of four places in flight together.
template <class Load, class Store>
__device__ __forceinline__ void move_pages(int64_t begin, int64_t end, int step, Load load, Store store) {
    for (int64_t j = begin; j < end; j += 4 * step) {
        int32_t page[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (j + i * step < end) page[i] = load(j + i * step);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (j + i * step < end) store(j + i * step, page[i]);
    }
}

__global__ void __launch_bounds__(kMapThreads) kv_map_kernel(const MapArgs a) {
    extern __shared__ int32_t s_rows[];  // need [B], held [B], off [B]
    __shared__ uint64_t s_warp[kMapWarps];
    __shared__ int32_t s_taken;
    int32_t *s_need = s_rows, *s_held = s_rows + a.B, *s_off = s_rows + 2 * a.B;
    const int tid = threadIdx.x, lane = tid & 31;
    const int cta = blockIdx.x, ctas = gridDim.x;  // the grid is one cluster
    auto owner = [&](int b) { return (b >> 5) % ctas; };
    auto sync = [&] {
        if (ctas == 1) {
            __syncthreads();
        } else {
            cluster_arrive_release();
            cluster_wait_acquire();
        }
    };
    pdl_wait();
    pdl_trigger();
    const int32_t count = min(max(__ldcg(a.free_count), 0), a.pages);
    if (tid == 0) s_taken = 0;
    uint64_t carry = 0;
    for (int b0 = 0; b0 < a.B; b0 += kMapThreads) {
        const int b = b0 + tid;
        uint64_t v = 0;
        if (b < a.B) {
            const int64_t len = int64_t(__ldcg(a.lens + b)) + a.lens_add, nw = int64_t(__ldcg(a.new_lens + b)) + a.new_add;
            const int32_t held = __ldcg(a.held + b);
            const bool ok = len >= 0 && nw >= 0 && nw <= a.T && held >= 0 && held <= a.blocks;
            const int64_t need64 = (len + nw + (int64_t(1) << a.page_shift) - 1) >> a.page_shift;
            int32_t st = SWITCHSD_ROW_OK, need = -1;
            if (!ok) {
                st = SWITCHSD_ROW_BAD_LEN;
            } else if (need64 > a.blocks) {
                st = SWITCHSD_ROW_CAPACITY;
            } else {
                need = int32_t(need64);
                v = need < held ? uint64_t(uint32_t(held - need)) : uint64_t(uint32_t(need - held)) << 32;
            }
            s_need[b] = need;
            s_held[b] = held;
            if (a.status && owner(b) == cta) a.status[b] = st;
        }
        uint64_t total;
        const uint64_t ex = carry + block_scan(v, s_warp, total);
        if (b < a.B) s_off[b] = s_need[b] < s_held[b] ? int32_t(uint32_t(ex)) : int32_t(min(ex >> 32, uint64_t(0x7fffffff)));
        carry += total;
    }
    __syncthreads();
    const int32_t n = int32_t(min(int64_t(count) + int64_t(uint32_t(carry)), int64_t(a.pages)));  // on the stack before the takes
    if (cta == 0) {
        int32_t taken = 0;
        for (int b = tid; b < a.B; b += kMapThreads) {
            if (s_need[b] <= s_held[b] || s_need[b] < 0) continue;  // (a bad row's held may be anything)
            const int64_t end = int64_t(s_off[b]) + (s_need[b] - s_held[b]);
            if (end <= n) taken = max(taken, int32_t(end));
        }
        taken = __reduce_max_sync(kFull, taken);
        if (lane == 0 && taken > 0) atomicMax(&s_taken, taken);
    }
    // The warps of a row: as many as there are for each, so that a few rows' long moves are not one warp's.
    const int mine = (a.B / (32 * ctas)) * 32 + min(max(a.B % (32 * ctas) - 32 * cta, 0), 32);  // this CTA's rows
    int share = 0;  // log2 of a row's warps
    while (share < 5 && (min(mine, 32) << (share + 1)) <= kMapWarps) ++share;
    const int part = (tid >> 5) & ((1 << share) - 1), step = kWarp << share;
    auto row_of = [&](int i) { return (i >> 5) * 32 * ctas + 32 * cta + (i & 31); };  // this CTA's i-th row
    const int first = tid >> (5 + share), rows_step = kMapWarps >> share;
    // 1. Rows that give pages back.
    for (int i = first; i < mine; i += rows_step) {
        const int b = row_of(i);
        const int32_t need = s_need[b], held = s_held[b];
        if (need < 0 || need >= held) continue;
        int32_t *row = a.table + size_t(b) * a.blocks;
        const int64_t at0 = int64_t(count) + s_off[b] - need;
        move_pages(
            need + part * kWarp + lane, held, step, [&](int64_t j) { return __ldcg(row + j); },
            [&](int64_t j, int32_t page) {
                if (at0 + j < a.pages) a.free_list[at0 + j] = page;
                row[j] = -1;
            });
    }
    sync();
    // 2. Rows that take pages: the i-th asked for is the i-th from the top.
    for (int i = first; i < mine; i += rows_step) {
        const int b = row_of(i);
        const int32_t need = s_need[b], held = s_held[b];
        const bool fits = need >= 0 && (need <= held || int64_t(s_off[b]) + (need - held) <= n);
        // (over new_lens itself, perhaps: every CTA has read it, and the slots read the rows' that keep it)
        if (a.granted && part == 0 && lane == 0) a.granted[b] = fits ? __ldcg(a.new_lens + b) : -1 - a.new_add;
        if (need < 0) continue;
        if (need > held) {
            if (!fits) {
                if (part == 0 && lane == 0 && a.status) a.status[b] = SWITCHSD_ROW_CAPACITY;
                continue;
            }
            int32_t *row = a.table + size_t(b) * a.blocks;
            const int64_t at0 = int64_t(n) - 1 - s_off[b] + held;
            move_pages(
                held + part * kWarp + lane, need, step, [&](int64_t j) { return __ldcg(a.free_list + (at0 - j)); },
                [&](int64_t j, int32_t page) {
                    row[j] = page;
                    a.free_list[at0 - j] = -1;
                });
        }
        if (part == 0 && lane == 0) a.held[b] = need;
    }
    sync();
    if (cta == 0 && tid == 0) *a.free_count = n - s_taken;
    // 3. Slots of this CTA's rows.
    if (a.slots) {
        for (int64_t k = tid; k < int64_t(mine) * a.T; k += kMapThreads) {  // (k passes 2^31 with a step of nearly as many tokens)
            const int i = int(uint32_t(k) / uint32_t(a.T)), t = int(uint32_t(k) - uint32_t(i) * uint32_t(a.T)), b = row_of(i);
            const int32_t need = s_need[b], held = s_held[b];
            int32_t slot = -1;
            if (need >= 0 && (need <= held || int64_t(s_off[b]) + (need - held) <= n) && t < __ldcg(a.new_lens + b) + a.new_add) {
                const int32_t p = __ldcg(a.lens + b) + a.lens_add + t;
                const int32_t page = __ldcg(a.table + size_t(b) * a.blocks + (p >> a.page_shift));
                slot = (page << a.page_shift) + (p & ((1 << a.page_shift) - 1));
            }
            a.slots[size_t(b) * a.T + t] = slot;
        }
    }
}

}  // namespace switchsd

using namespace switchsd;

extern "C" int switchsd_kv_map(const switchsd_kv_map_params *p) { return switchsd_kv_map_granted(p, nullptr); }

extern "C" int switchsd_kv_map_granted(const switchsd_kv_map_params *p, int32_t *granted) {
    if (!p || !p->lens || !p->new_lens || !p->block_table || !p->held || !p->free_list || !p->free_count) return SWITCHSD_ERR_ARG;
    if (p->B < 1 || p->B > SWITCHSD_MAP_ROWS || p->T < 1 || p->blocks < 1 || p->pages < 1 || !kv4_page_ok(p->page)) return SWITCHSD_ERR_SHAPE;
    if (int64_t(p->pages) * p->page > 0x7fffffff || int64_t(p->B) * p->T > 0x7fffffff || int64_t(p->B) * p->blocks > 0x7fffffff)
        return SWITCHSD_ERR_SHAPE;
    MapArgs a;
    a.lens = p->lens;
    a.new_lens = p->new_lens;
    a.table = p->block_table;
    a.held = p->held;
    a.free_list = p->free_list;
    a.free_count = p->free_count;
    a.slots = p->slots;
    a.status = p->status;
    a.granted = granted;
    a.B = p->B;
    a.T = p->T;
    a.blocks = p->blocks;
    a.pages = p->pages;
    a.page_shift = log2_of(p->page);
    a.lens_add = p->lens_add;
    a.new_add = p->new_add;
    const size_t smem = size_t(p->B) * 3 * sizeof(int32_t);
    static bool attr_done[64] = {false};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return SWITCHSD_ERR_CUDA;
    if (dev < 0 || dev >= 64 || !attr_done[dev]) {
        if (cudaFuncSetAttribute(kv_map_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SWITCHSD_MAP_ROWS * 12) != cudaSuccess)
            return SWITCHSD_ERR_CUDA;
        if (dev >= 0 && dev < 64) attr_done[dev] = true;
    }
    const unsigned ctas = unsigned(p->B < 32 * kMapCtas ? (p->B + 31) / 32 : kMapCtas);
    const cudaError_t e = launch_pdl(kv_map_kernel, dim3(ctas), dim3(kMapThreads), smem, static_cast<cudaStream_t>(p->stream), ctas, a);
    return e == cudaSuccess ? SWITCHSD_OK : SWITCHSD_ERR_CUDA;
}
