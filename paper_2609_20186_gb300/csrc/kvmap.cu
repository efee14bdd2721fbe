// kvmap.cu -- switchsd_kv_map: block tables and slot maps of a paged cache from the rows' device lengths.
//
// Two exclusive prefix sums over the rows decide everything: of the pages that rows give back (their places on the
// stack) and of the pages that rows ask for (their distance from its top).  A row either gives or asks, so both
// sums ride in one 64-bit scan.
#include "kv4.cuh"

namespace switchsd {

constexpr int kMapThreads = 1024;
constexpr int kMapWarps = kMapThreads / kWarp;

struct MapArgs {
    const int32_t *lens, *new_lens;
    int32_t *table, *held, *free_list, *free_count, *slots, *status;
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

__global__ void __launch_bounds__(kMapThreads) kv_map_kernel(const MapArgs a) {
    extern __shared__ int32_t s_rows[];  // need [B], held [B], off [B]
    __shared__ uint64_t s_warp[kMapWarps];
    __shared__ int32_t s_taken;
    int32_t *s_need = s_rows, *s_held = s_rows + a.B, *s_off = s_rows + 2 * a.B;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
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
            if (a.status) a.status[b] = st;
        }
        uint64_t total;
        const uint64_t ex = carry + block_scan(v, s_warp, total);
        if (b < a.B) s_off[b] = s_need[b] < s_held[b] ? int32_t(uint32_t(ex)) : int32_t(min(ex >> 32, uint64_t(0x7fffffff)));
        carry += total;
    }
    __syncthreads();
    const int32_t n = int32_t(min(int64_t(count) + int64_t(uint32_t(carry)), int64_t(a.pages)));  // on the stack before the takes
    // 1. Rows that give pages back, a warp a row.
    for (int b = warp; b < a.B; b += kMapWarps) {
        const int32_t need = s_need[b], held = s_held[b];
        if (need < 0 || need >= held) continue;
        int32_t *row = a.table + size_t(b) * a.blocks;
        for (int32_t j = need + lane; j < held; j += kWarp) {
            const int32_t at = count + s_off[b] + (j - need);
            if (at < a.pages) a.free_list[at] = __ldcg(row + j);
            row[j] = -1;
        }
    }
    __syncthreads();
    // 2. Rows that take pages: the i-th asked for is the i-th from the top.
    for (int b = warp; b < a.B; b += kMapWarps) {
        const int32_t need = s_need[b], held = s_held[b];
        if (need < 0) continue;
        if (need > held) {
            const int64_t end = int64_t(s_off[b]) + (need - held);
            if (end > n) {
                __syncwarp();
                if (lane == 0) {
                    s_need[b] = -1;
                    if (a.status) a.status[b] = SWITCHSD_ROW_CAPACITY;
                }
                continue;
            }
            int32_t *row = a.table + size_t(b) * a.blocks;
            for (int32_t j = held + lane; j < need; j += kWarp) {
                const int32_t at = n - 1 - (s_off[b] + (j - held));
                row[j] = __ldcg(a.free_list + at);
                a.free_list[at] = -1;
            }
            if (lane == 0) atomicMax(&s_taken, int32_t(end));
        }
        if (lane == 0) a.held[b] = need;
    }
    __syncthreads();
    if (tid == 0) *a.free_count = n - s_taken;
    // 3. Slots.
    if (a.slots) {
        for (int i = tid; i < a.B * a.T; i += kMapThreads) {
            const int b = i / a.T, t = i - b * a.T;
            int32_t slot = -1;
            if (s_need[b] >= 0 && t < __ldcg(a.new_lens + b) + a.new_add) {
                const int32_t p = __ldcg(a.lens + b) + a.lens_add + t;
                const int32_t page = __ldcg(a.table + size_t(b) * a.blocks + (p >> a.page_shift));
                slot = (page << a.page_shift) + (p & ((1 << a.page_shift) - 1));
            }
            a.slots[i] = slot;
        }
    }
}

}  // namespace switchsd

using namespace switchsd;

extern "C" int switchsd_kv_map(const switchsd_kv_map_params *p) {
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
    const cudaError_t e = launch_pdl(kv_map_kernel, dim3(1), dim3(kMapThreads), smem, static_cast<cudaStream_t>(p->stream), 0u, a);
    return e == cudaSuccess ? SWITCHSD_OK : SWITCHSD_ERR_CUDA;
}
