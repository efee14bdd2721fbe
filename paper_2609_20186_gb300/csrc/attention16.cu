// attention16.cu -- switchsd_kv16_attention: attention of a step's new tokens over the 16-bit paged cache, on tcgen05.
//
// Work.  The query rows of a row and key head -- its new tokens times the query heads that share the key head -- are cut
// into tiles of whole tokens, up to 256 rows; an item is one such tile over the keys that its last token sees, and its unit
// of work is 128 keys.  The units of all items, in order of rows, key heads and tiles, are dealt out evenly over a CTA an
// SM (the lengths are on the device; every CTA adds them up itself): a CTA takes a contiguous range, which may begin and
// end inside an item.  An item that one CTA holds whole is written out at once; the others leave partial results that a
// second kernel joins in order.
//
// A CTA has two slots, each with four warps for 128 query rows (a thread a row), its scores S = Q K^T and its output
// O = P V in tensor memory.  A tile of more than 128 rows has half of them in each slot, and both slots take every unit; a
// smaller one is in both slots, which take units in turn and join at the end.  While one slot's warps turn scores into
// weights, the tensor cores work for the other.  Further warps: one goes through the CTA's runs of units ahead of the others
// and brings their queries, one fetches tiles of keys and values through a ring (TMA, 128-byte swizzle, a box a page), one
// issues the products, one looks after the values' tiles.  So the next run's scores are computed while a slot's warps still
// write the last one's output.
//
// Numbers.  The operands are the cache's and the queries' own numbers, products exact, S and O in binary32.  P takes S's
// place in tensor memory, in the cache's type, since both operands of a product have one: weights are relative to a
// reference that may lag the largest score (kLagUp), so that O is scaled seldom, f16 weights 2^11 higher so that few are
// below its normal numbers; scores may be of any size (far_units).  Their sum is of the unrounded weights, in binary32.
//
// What a token does not see: scores are replaced before their maximum is taken.  Of the values, what no row of the tile sees
// (past its last token, without a page) is cleared in shared memory; among the values that some rows see and others do
// not, numbers that are not finite would reach the others as 0 * inf: they are cleared too, and added to the rows that see
// them at the end.
//
// Bound.  One token a row and up to a draft's: memory.  64 rows of 8K to 32K tokens, 8 key heads x 128, one token each:
// 785 us, 5.4 GB, all of a copy's rate; 1 to 17 tokens over 2K to 8K: 218 us (91 %), of which 6 are the join.  Chunks: 2 rows
// of 2048 tokens over 30K, 32 query heads: 1370 us, 1.55 PFLOP/s, 80 % of what a library's product reaches in a short run and
// 91 % of what it sustains.  The tensor pipe is active 75 % of the time; what it waits for is the chain of barriers between a
// slot's scores, weights and products, some 3000 cycles a unit, 1800 of them the rows' warps' (loads 240, maxima 500, weights
// 1000), and the warp that issues the products has one for both slots (100 to 200 cycles a wait).  It is not the exponentials:
// without them the time is the same.  16 rows of up to 500 tokens with heads of 64: 108 us, 4 times its products' time,
// since the chain is as long for a product of half the size, and a run has few units for its queries, masks and output (2 us a
// run); 10 us pass before the first scores.  One token over 2K: 12.8 us, latency (the dealing, queries, first tiles, and 4
// for the second launch).
//
// Why so.  Two slots: with one, the tensor cores wait while scores become weights.  Products issued by a warp that stays
// together: 1874 -> 1515 us for the chunks.  The warps that help are the first ones, so that the slots' registers are whole
// warpgroups': 1515 -> 1449.  Runs and queries ahead, by a warp of their own: 256 -> 229 us for the drafts.
// Not kept: weights before the unit's maximum is known, put right afterwards (chunks of 500 tokens 182 against 162); looking
// for the next scores before the second half of the weights (1610 against 1449); loading the scores a second time to have
// fewer registers (1813); sums and products one by one instead of packed in pairs (1505); three places for scores where heads
// have 64 dimensions (194 against 162); a quarter of the exponentials by a polynomial (1523 against 1440); maxima of the first
// half of the scores while the others are loaded (1519 against 1425); a warp of its own for each slot's products (1642 against
// 1425, since the slots fall into step; 791 against 801 for one token a row); waits that poll instead of sleeping (1472).
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <cstdlib>

#include "attention.cuh"
#include "tc.cuh"

namespace switchsd {

constexpr int kSlotRows = 128;              // query rows of a slot: the MMA's M
constexpr int kTileRows = 2 * kSlotRows;
constexpr int kUnitKeys = 128;
constexpr int kSlotThreads = kSlotRows, kSlotWarps = kSlotThreads / kWarp;
constexpr int kMmaWarp16 = 0, kFetchWarp16 = 1, kValueWarp16 = 2, kRunWarp = 3, kFirstSlotWarp = 4;
constexpr int kThreads16 = (2 * kSlotWarps + 4) * kWarp;
// Registers a thread of the two slots' warpgroups and of the third: 384 threads are launched with 168 each, and the shares
// add up to the same.  (176 / 152 a thread: 1474 us for chunks, 134 for chunks of 500 tokens; 216 / 72: 1488, 132; these: 1463, 130.)
constexpr int kSlotRegs = 192, kOtherRegs16 = 120;
static_assert(2 * kSlotRegs + kOtherRegs16 == 3 * 168, "what two warpgroups gain the third gives");
constexpr int kMaxCtas16 = 160;
constexpr int kPartExtra = 8;               // of a partial result's row: reference and sum, and room for rows of whole 32 bytes
constexpr int kReady = 8;                   // units whose values are on their way, at most (a ring's tiles are fewer)
constexpr int kRuns = 8;                    // runs between the first and the last of the warps, at most
// Units that a run costs beside its own when the units are dealt out: queries, masks, output.  (0: 232 us for drafts, 142 for
// chunks of 500 tokens; 1: 226, 130; 2: 224, 128; 4: 223, 127, but 14.2 instead of 13.4 for one token over 2K.)
constexpr int kRunCost = 2;
constexpr int kBlock16 = 128 * 128;         // 128 rows of one swizzle row: an operand's 64 elements
constexpr int kColumns16 = 512;             // tensor memory: S 2 x 128, O 2 x 128
// log2 of the weight of a score at the reference, and of one that is as large as can be without a new reference.
template <bool F16>
constexpr float kUp = F16 ? 11.f : 0.f;
template <bool F16>
constexpr float kLagUp = F16 ? 15.f : 8.f;
constexpr float kFar = 4194304.f;           // 2^22: the rounding of references of this size and more would show in the weights

struct Attn16Args : AttnArgs {
    int32_t tokens;  // of a tile: kTileRows / group
};

template <int D>
struct Smem16 {
    static constexpr int kQ = (D / 64) * kBlock16;      // a slot's queries: [D / 64][128 rows][128 bytes]
    static constexpr int kTile = (D / 64) * kBlock16;   // 128 keys or values: [D / 64][128 tokens][128 bytes]
    static constexpr int kQueries = D == 128 ? 2 : 4;   // slots' queries in shared memory
    static constexpr int kStages = D == 128 ? 5 : 10;
    static constexpr int bytes = 1024 + kQueries * kQ + kStages * kTile;
};

// K-major operands (sw128_desc), and V: [D / 64][token][64], the contracted axis outermost; groups of eight tokens are 1024
// bytes apart, the other 64 dimensions kBlock16.
__device__ __forceinline__ uint64_t value_desc(uint32_t saddr) {
    return uint64_t((saddr & 0x3FFFFu) >> 4) | (uint64_t(kBlock16 >> 4) << 16) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
}
// Instruction descriptor: binary32 sums, M = 128; `values`: B with the contracted axis outermost.
template <bool F16>
__device__ constexpr uint32_t idesc16(int N, bool values) {
    return f16_idesc(N) | (F16 ? 0u : (1u << 7) | (1u << 10)) | (values ? 1u << 16 : 0u);
}

// The products and commits of a warp that stays together: its threads run the same loop on the same numbers, and the leader's
// instructions alone take effect.  A loop of one thread's has its descriptors in ordinary registers, from where each product
// moves them at 100 cycles a product.
__device__ __forceinline__ uint32_t elect_leader() {
    uint32_t leader;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "elect.sync _|p, 0xffffffff;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(leader));
    return leader;
}
__device__ __forceinline__ void lead_mma_ss(uint32_t leader, uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, bool acc) {
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "setp.ne.b32 q, %5, 0;\n"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
        "}\n" ::"r"(d),
        "l"(da), "l"(db), "r"(idesc), "r"(uint32_t(acc)), "r"(leader)
        : "memory");
}
__device__ __forceinline__ void lead_mma_ts(uint32_t leader, uint32_t d, uint32_t ta, uint64_t db, uint32_t idesc, bool acc) {
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "setp.ne.b32 q, %5, 0;\n"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
        "}\n" ::"r"(d),
        "r"(ta), "l"(db), "r"(idesc), "r"(uint32_t(acc)), "r"(leader)
        : "memory");
}
__device__ __forceinline__ void lead_commit(uint32_t leader, uint64_t *bar) {
    asm volatile(
        "{\n"
        ".reg .pred q;\n"
        "setp.ne.b32 q, %1, 0;\n"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n"
        "}\n" ::"r"(smem_addr(bar)), "r"(leader)
        : "memory");
}
__device__ __forceinline__ void lead_arrive(uint32_t leader, uint64_t *bar) {
    asm volatile(
        "{\n"
        ".reg .pred q;\n"
        "setp.ne.b32 q, %1, 0;\n"
        "@q mbarrier.arrive.shared::cta.b64 _, [%0];\n"
        "}\n" ::"r"(smem_addr(bar)), "r"(leader)
        : "memory");
}

__device__ __forceinline__ void tma_load_4d(void *dst, const CUtensorMap *map, int32_t x, int32_t y, int32_t z, int32_t w, uint64_t *bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n" ::"r"(smem_addr(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_addr(bar))
        : "memory");
}

// 32 bytes; p is a multiple of 32.
__device__ __forceinline__ void store32(void *p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
__device__ __forceinline__ void tmem_st2(uint32_t taddr, uint32_t a, uint32_t b) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x2.b32 [%0], {%1, %2};\n" ::"r"(taddr), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ void tmem_ld2(uint32_t taddr, uint32_t (&r)[2]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x2.b32 {%0, %1}, [%2];\n" : "=r"(r[0]), "=r"(r[1]) : "r"(taddr));
}

// sum over i < n of floor((c + a i) / 128): the sum of the numbers less that of their remainders, which repeat.
__device__ __forceinline__ int64_t sum_of_units(int64_t c, int32_t a, int64_t n) {
    const int32_t g = min(128, a & -a), log_period = 8 - __ffs(g), period = 1 << log_period, some = int32_t(n) & (period - 1);
    int64_t rest = (n >> log_period) * (int64_t(period) * (c & (g - 1)) + (int64_t(g) * period * (period - 1) >> 1));
    int32_t r = int32_t(c & 127);
    for (int32_t i = 0; i < some; ++i, r = (r + a) & 127) rest += r;
    return (n * c + a * (n * (n - 1) / 2) - rest) >> 7;
}

// n / d, n below 2^63: 32 bits where they are enough.
__device__ __forceinline__ int64_t quotient(int64_t n, int64_t d) {
    return ((n | d) >> 32) == 0 ? int64_t(uint32_t(n) / uint32_t(d)) : n / d;
}

// A run of units of one item.
struct Run {
    int b, hk, rt;
    int32_t len, token0, tokens, keys;  // of the tile: its first token, tokens, and keys that its last one sees
    int32_t first, n, units, part;      // part: which of the CTA's two partial results it may leave
    int32_t parts;                      // CTAs that hold units of the item
};
// The runs of a CTA's range, in order, but that one which begins inside an item comes last: the CTAs that share an item's
// keys then go through them side by side, and what one has fetched the others find in L2.
struct Runs {
    int64_t u, total;    // units and runs' costs before the next run, in all
    int32_t takers;
    int b, hk, rt;
    int32_t skip;        // of the first item: what lies before the range
    int64_t left;        // what is left of the range
    int32_t len, nw;     // of row b
    bool begun, held;
    Run late;
    __device__ int holder(int64_t at) const { return int(quotient((at + 1) * takers - 1, total)); }  // the CTA whose range has it
    __device__ bool take(const Attn16Args &a, Run &s) {
        while (left > 0) {
            const int tiles = (nw + a.tokens - 1) / a.tokens;
            if (rt >= tiles) {
                rt = 0;
                if (nw == 0 || ++hk == a.Hkv) {
                    hk = 0;
                    ++b;
                    row_lengths(a, b, len, nw);
                }
                continue;
            }
            s.b = b;
            s.hk = hk;
            s.rt = rt++;
            s.len = len;
            s.token0 = s.rt * a.tokens;
            s.tokens = min(a.tokens, nw - s.token0);
            s.keys = len + s.token0 + s.tokens;
            s.units = (s.keys + kUnitKeys - 1) / kUnitKeys;
            const int32_t taken = int32_t(min(int64_t(kRunCost + s.units - skip), left));
            s.first = max(0, skip - kRunCost);
            s.n = skip + taken - kRunCost - s.first;
            s.part = 1;
            const int64_t unit0 = u - skip + kRunCost;  // the item's first
            s.parts = holder(unit0 + s.units - 1) - holder(unit0) + 1;
            u += taken;
            skip = 0;
            left -= taken;
            if (s.n > 0) return true;  // (else the range ends before the item's first unit)
        }
        return false;
    }
    __device__ bool next(const Attn16Args &a, Run &s) {
        if (!begun) {
            begun = true;
            if (!take(a, s)) return false;
            s.part = 0;
            if (s.first == 0 || left == 0) return true;
            late = s;
            held = true;
        }
        if (take(a, s)) return true;
        if (!held) return false;
        held = false;
        s = late;
        return true;
    }
};

// The CTA's range.  Also: statuses (CTA 0), and the CTA's partial results marked as none.  All threads call it.  s_pre:
// kThreads16 + 2 numbers.
__device__ __forceinline__ void deal_runs(const Attn16Args &a, int64_t *s_pre, Runs &runs) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x, ctas = int(gridDim.x);
    const int per = (a.B + kThreads16 - 1) / kThreads16;  // rows of a thread
    auto before_tile = [&](int32_t len, int32_t nw, int rt) -> int64_t {  // units and costs of a key head's tiles before rt
        const int whole = nw / a.tokens;
        const int64_t c = int64_t(len) + a.tokens + kUnitKeys - 1;
        return int64_t(rt) * kRunCost + (whole && rt ? sum_of_units(c, a.tokens, min(rt, whole)) : 0) +
               (rt > whole ? (int64_t(len) + nw + kUnitKeys - 1) / kUnitKeys : 0);
    };
    int32_t len = 0, nw = 0;
    auto units_of = [&](int row) -> int64_t {  // of a key head
        const bool ok = row_lengths(a, row, len, nw);
        if (a.status && cta == 0) a.status[row] = ok ? SWITCHSD_ROW_OK : SWITCHSD_ROW_BAD_LEN;
        return nw ? before_tile(len, nw, (nw + a.tokens - 1) / a.tokens) : 0;
    };
    int64_t mine = 0, n = 0;
    for (int i = 0; i < per; ++i)
        if (tid * per + i < a.B) mine += (n = units_of(tid * per + i)) * a.Hkv;
    int64_t x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(kFull, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) s_pre[warp] = x;
    __syncthreads();
    int64_t total = 0, before = x - mine;  // of all rows, of those before the thread's
#pragma unroll
    for (int w = 0; w < kThreads16 / kWarp; ++w) {
        const int64_t y = s_pre[w];
        total += y;
        if (w < warp) before += y;
    }
    const int64_t takers = min(total, int64_t(ctas));  // CTAs with a range
    const int64_t u = cta < takers ? quotient(total * cta, takers) : total, u_end = cta < takers ? quotient(total * (cta + 1), takers) : total;
    if (tid < 2) a.desc[2 * cta + tid] = make_int4(-1, 0, 0, 0);
    int64_t *s_at = s_pre + kThreads16 / kWarp;
    if (u < u_end && u >= before && u < before + mine) {
        int64_t at = before;
        int row = tid * per;
        if (per > 1)
            for (;; ++row) {
                n = units_of(row);
                if (u < at + n * a.Hkv) break;
                at += n * a.Hkv;
            }
        const int64_t hk = quotient(u - at, n), off = u - at - hk * n;
        int lo = 0, hi = (nw + a.tokens - 1) / a.tokens;  // the last tile with no more than `off` units before it
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            (before_tile(len, nw, mid) <= off ? lo : hi) = mid;
        }
        s_at[0] = row;
        s_at[1] = hk;
        s_at[2] = lo;
        s_at[3] = off - before_tile(len, nw, lo);
        s_at[4] = (int64_t(len) << 32) | nw;
    }
    __syncthreads();
    runs.b = int(s_at[0]);
    runs.hk = int(s_at[1]);
    runs.rt = int(s_at[2]);
    runs.skip = int32_t(s_at[3]);
    runs.len = int32_t(s_at[4] >> 32);
    runs.nw = int32_t(s_at[4]);
    runs.left = u < u_end ? u_end - u : 0;
    runs.u = u;
    runs.total = total;
    runs.takers = int32_t(takers);
    runs.begun = runs.held = false;
}

// Zeros for the tokens that are not there, by warp w of so many: it looks at 32 tokens together and fills a part of each, 512
// bytes or more.
__device__ __forceinline__ void fill_absent(const Attn16Args &a, uint32_t w, uint32_t warps) {
    const int lane = threadIdx.x & 31;
    const uint32_t all = uint32_t(a.B) * uint32_t(a.T), groups = (all + kWarp - 1) / kWarp;  // (below 2^31)
    const uint32_t row16 = uint32_t(a.Hq) * uint32_t(a.dim / 8);                             // 16-byte pieces of a token's output
    const uint32_t cuts = max(1u, min(warps / groups, row16 / kWarp)), cut = (row16 + cuts - 1) / cuts;
    for (; w < groups * cuts; w += warps) {
        const uint32_t j0 = w / cuts * kWarp, j = j0 + lane, b = j / uint32_t(a.T), e0 = w % cuts * cut, e1 = min(e0 + cut, row16);
        int32_t len, nw = a.T;
        if (j < all) row_lengths(a, int(b), len, nw);
        for (uint32_t gone = __ballot_sync(kFull, int(j - b * a.T) >= nw); gone; gone &= gone - 1) {
            uint4 *o = reinterpret_cast<uint4 *>(a.out) + size_t(j0 + __ffs(int(gone)) - 1) * row16;
            for (uint32_t e = e0 + lane; e < e1; e += kWarp) o[e] = make_uint4(0, 0, 0, 0);
        }
    }
}

// Bits of the keys from `key` on that a row sees whose last visible one is `limit`, among 32 of a unit.
__device__ __forceinline__ uint32_t seen_of(uint32_t there, int32_t limit, int32_t key) {
    const int32_t ahead = limit - key;
    return there & (ahead >= 31 ? 0xffffffffu : ahead < 0 ? 0u : (2u << ahead) - 1u);
}

// A row's reference and sum of weights follow a unit's largest score mx (times the scale), and so does O, where there is one.  Returns
// whether a reference of the warp's has changed.  All of a warp.
template <bool F16, int D>
__device__ __forceinline__ bool follow(float mx, float &ref, float &l, uint32_t out, bool has_out) {
    float corr = 1.f;
    if (mx > __fadd_rd(ref, kLagUp<F16>)) {  // (both rounded so that weights stay small: f16 has none beyond 2^15)
        const float to = __fsub_ru(mx, kUp<F16>);
        corr = exp2_approx(ref - to);
        ref = to;
        l *= corr;
    }
    if (!__any_sync(kFull, corr != 1.f)) return false;
    if (has_out)
#pragma unroll 1
        for (int e = 0; e < D; e += 16) {
            uint32_t w[16];
            tmem_ld16(out + e, w);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 16; ++j) w[j] = __float_as_uint(__uint_as_float(w[j]) * corr);
            tmem_st16(out + e, w);
        }
    return true;
}

// A row's units from k on, of which the first one's scores are there, where references of the warp's are far: exponents are of
// products rounded as the reference's was, since an exact one lies up to half of a step of the reference beside it, and weights of
// the largest score itself would be infinite or 0.  Little code, in a place of its own: chunks of 500 tokens 108.3 us with it, 105.7
// without, the other cases alike.  (Where these took 114.5 and chunks 1434 without any such form: a branch in the loop 119.5 and 1460;
// a second form of the whole loop 119, 1428; exponents of score less reference, which need no such form but an addition more a pair,
// 122, 1515.)
struct FarRow {
    float ref, l;
    int32_t k;
    uint32_t i;
    bool ok;
};
template <bool F16, int D>
__device__ __forceinline__ FarRow far_units(FarRow r, uint32_t scores, uint32_t out, int32_t n, int32_t step, int32_t k0, int32_t key0, int32_t limit, uint32_t unit0,
                                            float scale, const uint32_t (*exist)[4], uint64_t *s_full, uint64_t *p_half, uint64_t *p_full) {
    const float size = fabsf(scale);
    for (bool there_already = true; r.k < n; r.k += step, ++r.i) {
        if (!there_already) r.ok = tc_wait_warp(s_full, r.i & 1);
        there_already = false;
        if (!r.ok) break;
        tc_fence_after();
        const uint32_t *there = exist[(unit0 + uint32_t(r.k)) % kReady];
        auto scores_of = [&](int w, float (&v)[32]) {
            tmem_ld32(scores + 32 * w, v);
            const uint32_t see = seen_of(there[w], limit, key0 + r.k * kUnitKeys + 32 * w);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = (see >> e) & 1 ? (scale < 0.f ? -v[e] : v[e]) : -INFINITY;
        };
        float mx = -INFINITY, sum = 0.f, v[32];
#pragma unroll 1
        for (int w = 0; w < 4; ++w) {
            scores_of(w, v);
#pragma unroll
            for (int e = 0; e < 32; e += 2) mx = max3(mx, v[e], v[e + 1]);
        }
        follow<F16, D>(__fmul_rn(mx, size), r.ref, r.l, out, r.k != k0);
        const bool rounded = fabsf(r.ref) > kFar;
#pragma unroll 1
        for (int w = 0; w < 4; ++w) {
            uint32_t y[16];
            scores_of(w, v);
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = exp2_approx(rounded ? __fsub_rn(__fmul_rn(v[e], size), r.ref) : __fmaf_rn(v[e], size, -r.ref));
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                sum += v[2 * e] + v[2 * e + 1];
                y[e] = narrow2<F16>(v[2 * e], v[2 * e + 1]);
            }
            tmem_st16(scores + 16 * w, y);
            if (w == 1) {
                tmem_wait_st();
                tc_fence_before();
                warp_arrive(p_half);
            }
        }
        r.l += sum;
        tmem_wait_st();
        tc_fence_before();
        warp_arrive(p_full);
    }
    return r;
}

template <bool F16, int D>
__global__ void __launch_bounds__(kThreads16, 1) attn16_kernel(const __grid_constant__ CUtensorMap map, const Attn16Args a) {
    using S = Smem16<D>;
    constexpr int N = S::kStages, G = D / 64;
    constexpr int NQ = S::kQueries;
    extern __shared__ uint8_t smem_raw[];
    // A tile's arrival has a barrier by its unit and kind, not by its stage: a phase is then waited for by everyone who waits
    // on that barrier at all, before its next one can begin.  (A stage has keys and values in turn, and who waits for the values
    // only would take a phase of the keys that is still to come, or is over, for another.)
    __shared__ __align__(8) uint64_t full[2][kReady], ready[kReady], empty[N], run_full[kRuns], q_ready[NQ], q_free[NQ];
    __shared__ __align__(8) uint64_t s_full[2], p_half[2], p_full[2], o_done[2], met, taken, written, stopped;
    __shared__ __align__(16) uint32_t s_exist[kReady][4];  // of a unit: its keys that exist and whose page does
    __shared__ __align__(16) int4 s_run[kRuns][3];
    __shared__ uint32_t s_tmem, s_cleared[kRuns];          // s_cleared: a run (+ 1) with values that were not finite, by the run
    __shared__ int s_bad;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x;
    uint8_t *base = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    uint8_t *sm_q = base, *sm_kv = base + NQ * S::kQ;

    if (tid == 0) {
        for (int i = 0; i < N; ++i) mbar_init(&empty[i], 1);
        for (int i = 0; i < kReady; ++i) {
            mbar_init(&full[0][i], 1);
            mbar_init(&full[1][i], 1);
            mbar_init(&ready[i], 1);
        }
        for (int i = 0; i < kRuns; ++i) {
            mbar_init(&run_full[i], 1);
            s_cleared[i] = 0;
        }
        for (int i = 0; i < NQ; ++i) {
            mbar_init(&q_ready[i], 1);
            mbar_init(&q_free[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s_full[i], 2);  // the products, and the MMA warp: what it has seen of the other warps
            mbar_init(&o_done[i], 2);
            mbar_init(&p_half[i], kSlotWarps);
            mbar_init(&p_full[i], kSlotWarps);
        }
        mbar_init(&met, 2 * kSlotWarps);
        mbar_init(&taken, 2 * kSlotWarps);
        mbar_init(&written, 2 * kSlotWarps);
        mbar_init(&stopped, 1);
        fence_mbar_init();
        s_bad = 0;
    }
    if (warp == kMmaWarp16) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_addr(&s_tmem)), "r"(kColumns16) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    pdl_wait();
    pdl_trigger();
    Runs runs;
    deal_runs(a, reinterpret_cast<int64_t *>(sm_kv), runs);
    fence_proxy_async();  // (the ring's memory was just used)
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    // Every wait of this warp has ended in time.  After one that has not, the warp goes to the end, and no result counts.
    bool ok = true;
    Run s;
    // The CTA's r-th run; n = 0: there are no more.
    auto read_run = [&](uint32_t r) {
        ok = ok && tc_wait_warp(&run_full[r % kRuns], (r / kRuns) & 1);
        const int4 x = s_run[r % kRuns][0], y = s_run[r % kRuns][1], z = s_run[r % kRuns][2];
        s = Run{x.x, x.y, x.z, y.x, y.y, y.z, y.w, z.x, z.y, z.z, x.w, z.w};
        return ok && s.n > 0;
    };

    if (warp >= kFirstSlotWarp) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kSlotRegs));
        // ------------------------------------------------------------------------------------------- query rows
        const int slot = warp / kSlotWarps - 1, quarter = warp % kSlotWarps, place = tid % kSlotThreads;
        const uint32_t lanes = tmem + (uint32_t(32 * quarter) << 16), scores = lanes + uint32_t(slot * 128);
        const bool flip = a.scale < 0.f;
        // of a sum of products, for the binary logarithm; positive, so that what is masked stays -inf (2^-149 for 0: no score shows it)
        const float scale = a.scale == 0.f ? 0x1p-149f : fabsf(a.scale) * 1.4426950408889634f;
        uint32_t i = 0, done = 0, splits = 0, unit0 = 0;  // this slot's units and runs so far, the CTA's runs in both slots and units
        for (uint32_t nrun = 0; read_run(nrun); ++nrun, unit0 += uint32_t(s.n)) {
            const int rows = s.tokens * a.group;
            const bool split = rows <= kSlotRows;  // the tile is in both slots, which take units in turn
            const int row = split ? place : slot * kSlotRows + place, t = row / a.group, h = s.hk * a.group + row - t * a.group;
            const bool mine = row < rows, warp_mine = row - lane < rows;
            const int32_t limit = mine ? s.len + s.token0 + t : -1;
            float ref = kFloor, l = 0.f;
            const int step = split ? 2 : 1, k0 = split ? slot : 0;
            const uint32_t out = lanes + 256 + uint32_t(slot * 128);
            int32_t k = k0;
            bool far = false;
            for (; k < s.n; k += step, ++i) {
                const int32_t key0 = (s.first + k) * kUnitKeys;
                ok = ok && tc_wait_warp(&s_full[slot], i & 1);
                if (!ok) break;
                tc_fence_after();
                if (warp_mine) {
                    float v[kUnitKeys];
#pragma unroll
                    for (int w = 0; w < 4; ++w) tmem_ld32(scores + 32 * w, v + 32 * w);
                    const uint4 there = *reinterpret_cast<const uint4 *>(s_exist[(unit0 + uint32_t(k)) % kReady]);
                    tmem_wait_ld();
                    if (flip)
#pragma unroll
                        for (int e = 0; e < kUnitKeys; ++e) v[e] = -v[e];
                    if (key0 + kUnitKeys > s.len + s.token0 + 1 || (there.x & there.y & there.z & there.w) != 0xffffffffu) {
                        const uint32_t word[4] = {there.x, there.y, there.z, there.w};
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            const uint32_t see = seen_of(word[w], limit, key0 + 32 * w);
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[32 * w + e] = (see >> e) & 1 ? v[32 * w + e] : -INFINITY;
                        }
                    }
                    float top[8] = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
#pragma unroll
                    for (int e = 8; e < kUnitKeys; e += 2) top[(e >> 1) & 7] = max3(top[(e >> 1) & 7], v[e], v[e + 1]);
                    const float mx = __fmul_rn(max3(max3(top[0], top[1], top[2]), max3(top[3], top[4], top[5]), fmaxf(top[6], top[7])), scale);
                    if (follow<F16, D>(mx, ref, l, out, k != k0))  // (the scores' product came behind the last one of O)
                        far = __any_sync(kFull, mine && fabsf(ref) > kFar && ref > kFloor);  // (what is in rows that are not there is no one's)
                    if (__builtin_expect(far, 0)) break;
                    const uint64_t scale2 = pair_of(scale, scale), ref2 = pair_of(-ref, -ref);
                    uint64_t sum[2] = {0, 0};
#pragma unroll
                    for (int w = 0; w < 4; ++w) {  // 32 keys, in 16 columns
                        uint32_t y[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const float2 x = halves_of(fma_pair(pair_of(v[32 * w + 2 * e], v[32 * w + 2 * e + 1]), scale2, ref2));
                            const float p0 = exp2_approx(x.x), p1 = exp2_approx(x.y);
                            sum[e & 1] = add_pair(sum[e & 1], pair_of(p0, p1));
                            y[e] = narrow2<F16>(p0, p1);
                        }
                        tmem_st16(scores + 16 * w, y);
                        if (w == 1) {  // the product of the first half may begin
                            tmem_wait_st();
                            tc_fence_before();
                            warp_arrive(&p_half[slot]);
                        }
                    }
                    const float2 both = halves_of(add_pair(sum[0], sum[1]));
                    l += both.x + both.y;
                    tmem_wait_st();
                } else {
                    warp_arrive(&p_half[slot]);
                }
                tc_fence_before();
                warp_arrive(&p_full[slot]);
            }
            if (__builtin_expect(far, 0)) {
                const FarRow r = far_units<F16, D>(FarRow{ref, l, k, i, ok}, scores, out, s.n, step, k0, s.first * kUnitKeys, limit, unit0, flip ? -scale : scale, s_exist,
                                                   &s_full[slot], &p_half[slot], &p_full[slot]);
                ref = r.ref;
                l = r.l;
                i = r.i;
                ok = r.ok;
            }
            // --- the run's result -------------------------------------------------------------------------------
            if (k0 < s.n) {
                ok = ok && tc_wait_warp(&o_done[slot], done & 1);
                ++done;
            }
            if (!ok) break;
            tc_fence_after();
            float f = 1.f, f1 = 0.f;          // of this slot's output (or the first one's), and the second one's
            const bool two = split && s.n > 1;  // the second slot has an output too
            if (split) {
                // References and sums change hands in the scores' place, in one of two places in turn.  The second slot has
                // nothing to wait for in a run of one unit and puts its own down while the first one may still read what it
                // put down before: that is in the other place, and in the same one only behind `met` of the run between,
                // where the first slot arrives once it has read.
                const uint32_t hand = 2 * (splits & 1);
                if (warp_mine) {
                    tmem_st2(scores + hand, __float_as_uint(ref), __float_as_uint(l));
                    tmem_wait_st();
                }
                tc_fence_before();
                warp_arrive(&met);
                ok = tc_wait_warp(&met, splits & 1);
                ++splits;
                if (!ok) break;
                tc_fence_after();
                if (warp_mine) {
                    uint32_t other[2];
                    tmem_ld2(lanes + uint32_t((1 - slot) * 128) + hand, other);
                    tmem_wait_ld();
                    const float its_ref = __uint_as_float(other[0]), its_l = __uint_as_float(other[1]);
                    const float top = fmaxf(ref, its_ref), own = exp2_approx(ref - top), its = exp2_approx(its_ref - top);
                    f = slot == 0 ? own : its;
                    f1 = slot == 0 ? its : own;
                    l = slot == 0 ? l * f + its_l * f1 : its_l * f + l * f1;  // (the same for both)
                    ref = top;
                }
                tc_fence_before();
            }
            warp_arrive(&taken);
            const bool whole = s.first == 0 && s.n == s.units;
            const float inv = l == 0.f ? 0.f : 1.f / l;
            if (warp_mine) {
                const uint32_t from = split ? lanes + 256 : out;
                const int part = 2 * cta + s.part, d0 = split ? slot * (D / 2) : 0, d1 = split ? d0 + D / 2 : D;
                float *partial = a.part + (size_t(part) * kTileRows + row) * (D + kPartExtra);
                uint16_t *result = a.out + ((size_t(s.b) * a.T + s.token0 + t) * a.Hq + h) * D;
                const bool wide = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0;
                const int32_t cleared = s_cleared[nrun % kRuns] == nrun + 1 ? min(limit + 1, (s.first + s.n) * kUnitKeys) : 0;
// (as short as can be: what runs once a run is not in the instruction caches; unrolled by four, 128 us instead of 119 for chunks of 500)
#pragma unroll 1
                for (int d = d0; d < d1; d += 16) {
                    float v[16];
                    uint32_t w[16];
                    tmem_ld16(from + d, w);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] = __uint_as_float(w[j]) * f;
                    if (two) {
                        tmem_ld16(from + 128 + d, w);
                        tmem_wait_ld();
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] = fmaf(__uint_as_float(w[j]), f1, v[j]);
                    }
                    for (int32_t key = max(s.first * kUnitKeys, s.len + s.token0 + 1); key < cleared; ++key) {  // (seldom)
                        const int32_t page = __ldcg(a.table + size_t(s.b) * a.blocks + (key >> a.page_shift));
                        if (uint32_t(page) >= uint32_t(a.pages)) continue;
                        const size_t line = (((size_t(page) * 2 + 1) * a.Hkv + s.hk) << a.page_shift) + (key & ((1 << a.page_shift) - 1));
                        const uint16_t *src = reinterpret_cast<const uint16_t *>(a.cache) + line * D + d;
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const float x = widen1<F16>(__ldcg(src + j));
                            if (!(fabsf(x) < INFINITY)) v[j] += x;
                        }
                    }
                    // (every thread has a row of its own: a store's 32 pieces are sectors of as many lines, so they are whole ones)
                    if (mine && whole) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) w[j] = narrow2<F16>(v[2 * j] * inv, v[2 * j + 1] * inv);
                        if (wide) {
                            store32(result + d, *reinterpret_cast<uint32_t(*)[8]>(w));
                        } else {
                            reinterpret_cast<uint4 *>(result + d)[0] = make_uint4(w[0], w[1], w[2], w[3]);
                            reinterpret_cast<uint4 *>(result + d)[1] = make_uint4(w[4], w[5], w[6], w[7]);
                        }
                    } else if (mine) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) w[j] = __float_as_uint(v[j]);
                        store32(partial + d, *reinterpret_cast<uint32_t(*)[8]>(w));
                        store32(partial + d + 8, *reinterpret_cast<uint32_t(*)[8]>(w + 8));
                    }
                }
                if (!whole && mine && d0 == 0) {
                    partial[D] = ref;
                    partial[D + 1] = l;
                    if (tid == kFirstSlotWarp * kWarp) a.desc[part] = make_int4(s.b, s.hk, s.token0, (s.first == 0 ? kFirst : 0) | (rows << 3) | (s.parts << 16));
                }
            }
            tc_fence_before();
            warp_arrive(&written);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kOtherRegs16));
        if (warp == kFetchWarp16) {
            // --------------------------------------------------------------------------------------- fetching
            // Lane G q + g copies the 64 dimensions g of the unit's q-th run of tokens inside a page.
            const int run = min(kUnitKeys, 1 << a.page_shift), nruns = kUnitKeys / run, page_mask = (1 << a.page_shift) - 1;
            const int q = lane / G, g = lane - G * q;
            uint32_t unit = 0, issued = 0;  // units, tiles
            for (uint32_t nrun = 0; read_run(nrun); ++nrun) {
                auto find = [&](int32_t k) {  // the page of this lane's tokens in unit k of the run
                    const int32_t key = (s.first + k) * kUnitKeys + q * run;
                    return q < nruns && k < s.n && key < s.keys ? __ldcg(a.table + size_t(s.b) * a.blocks + (key >> a.page_shift)) : -1;
                };
                int32_t page = find(0);
                for (int32_t k = 0; ok && k < s.n; ++k, ++unit) {
                    const int32_t key0 = (s.first + k) * kUnitKeys, next = find(k + 1);
                    const bool good = uint32_t(page) < uint32_t(a.pages);
                    const uint32_t goods = __ballot_sync(kFull, good);
                    const uint32_t bytes = uint32_t(__popc(goods)) * uint32_t(run) * 128u;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t x = 2 * unit + half, st = x % N;
                        if (x >= N) ok = ok && tc_wait_warp(&empty[st], (x / N - 1) & 1);
                        if (!ok) break;
                        if (half == 0 && lane < 4) {
                            uint32_t word = 0;
                            for (int e = 0; e < 32; e += 16) {  // runs are multiples of 16 tokens
                                const int at = 32 * lane + e, left = s.keys - (key0 + at);
                                if ((goods >> (G * (at / run))) & 1) word |= (left >= 16 ? 0xffffu : left > 0 ? (1u << left) - 1u : 0u) << e;
                            }
                            s_exist[unit % kReady][lane] = word;
                        }
                        __syncwarp();
                        if (lane == 0) mbar_arrive_expect_tx(&full[half][unit % kReady], bytes);
                        __syncwarp();
                        if (good)
                            tma_load_4d(sm_kv + st * S::kTile + g * kBlock16 + q * run * 128, &map, 64 * g, (key0 + q * run) & page_mask,
                                        half * a.Hkv + s.hk, page, &full[half][unit % kReady]);
                        issued = x + 1;
                    }
                    page = next;
                }
            }
            // copies in flight write shared memory: it stays the CTA's until they have come (also where another warp gave up on them)
            for (uint32_t x = issued > N ? issued - N : 0; x < issued; ++x) (void)tc_wait(&full[x & 1][x / 2 % kReady], (x / 2 / kReady) & 1);
        } else if (warp == kMmaWarp16) {
            // --------------------------------------------------------------------------------------- the products
            uint32_t unit0 = 0, qx = 0, weights[2] = {0, 0};  // units and slots' queries so far, units whose weights a slot's product took
            const uint32_t leader = elect_leader(), tm = __shfl_sync(kFull, tmem, 0);
            const uint64_t dq0 = sw128_desc(smem_addr(sm_q)), dk0 = sw128_desc(smem_addr(sm_kv)), dv0 = value_desc(smem_addr(sm_kv));
            auto stage_of = [&](uint32_t x) { return uint64_t(x % N) * (S::kTile >> 4); };
            auto score = [&](int slot, uint32_t query, uint32_t unit, bool first) {  // S = Q K^T; first: of the unit
                if (first) ok = ok && tc_wait_warp(&full[0][unit % kReady], (unit / kReady) & 1);
                if (!ok) return;
                lead_arrive(leader, &s_full[slot]);
                tc_fence_after();
                const uint64_t dq = dq0 + uint64_t(query % NQ) * (S::kQ >> 4), dk = dk0 + stage_of(2 * unit);
#pragma unroll
                for (int e = 0; e < D / 16; ++e) {
                    const uint64_t step = uint64_t(((e >> 2) * kBlock16 + (e & 3) * 32) >> 4);
                    lead_mma_ss(leader, tm + slot * 128, dq + step, dk + step, idesc16<F16>(kUnitKeys, false), e != 0);
                }
                lead_commit(leader, &s_full[slot]);
            };
            auto product = [&](int slot, uint32_t unit, bool first, bool fresh) {  // O += P V, half of the keys as soon as their weights are there
                if (first) ok = ok && tc_wait_warp(&ready[unit % kReady], (unit / kReady) & 1);
                const uint64_t dv = dv0 + stage_of(2 * unit + 1);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    ok = ok && tc_wait_warp(half ? &p_full[slot] : &p_half[slot], weights[slot] & 1);
                    if (!ok) return;
                    tc_fence_after();
#pragma unroll
                    for (int e = half * (kUnitKeys / 32); e < (half + 1) * (kUnitKeys / 32); ++e)
                        lead_mma_ts(leader, tm + 256 + slot * 128, tm + slot * 128 + 8 * e, dv + uint64_t((e * 16 * 128) >> 4), idesc16<F16>(D, true), !fresh || e != 0);
                }
                ++weights[slot];
            };
            auto release = [&](uint32_t x) {
                if (ok) lead_commit(leader, &empty[x % N]);
            };
            auto finish = [&](int slot) {
                if (!ok) return;
                lead_arrive(leader, &o_done[slot]);
                lead_commit(leader, &o_done[slot]);
            };
            for (uint32_t nrun = 0; !a.give_up && __any_sync(kFull, read_run(nrun)); ++nrun) {
                const bool split = __any_sync(kFull, s.tokens * a.group <= kSlotRows);
                const int32_t n = __shfl_sync(kFull, s.n, 0);
                const uint32_t q0 = qx, q1 = split ? qx : qx + 1;
                qx = q1 + 1;
                ok = tc_wait_warp(&q_ready[q0 % NQ], (q0 / NQ) & 1) && (split || tc_wait_warp(&q_ready[q1 % NQ], (q1 / NQ) & 1));
                if (nrun > 0) ok = ok && tc_wait_warp(&taken, (nrun - 1) & 1);  // the scores' place
                const int step = split ? 2 : 1;
                for (int32_t k = 0; ok && k < n + step; ++k) {
                    if (k == step && nrun > 0) ok = tc_wait_warp(&written, (nrun - 1) & 1);  // the outputs' place
#pragma unroll
                    for (int slot = 0; slot < 2; ++slot) {
                        if (split && slot != (k & 1)) continue;
                        const bool first = split || slot == 0, frees = split || slot == 1;  // the first and the last to use the unit's tiles
                        if (k >= step) {
                            product(slot, unit0 + k - step, first, k - step < step);
                            if (frees) release(2 * (unit0 + k - step) + 1);
                            if (k >= n) finish(slot);
                        }
                        if (k < n) {
                            score(slot, slot ? q1 : q0, unit0 + k, first);
                            if (frees) release(2 * (unit0 + k));
                            if (frees && k == n - 1 && ok) {
                                lead_commit(leader, &q_free[q0 % NQ]);
                                if (!split) lead_commit(leader, &q_free[q1 % NQ]);
                            }
                        }
                    }
                }
                unit0 += uint32_t(n);
            }
            // what is in flight reads shared and tensor memory (the rows' threads wait for the last product too, unless they gave up)
            lead_commit(leader, &stopped);
            (void)tc_wait(&stopped, 0);
        } else if (warp == kValueWarp16) {
            // --------------------------------------------------------------------------------------- values that not every row sees
            uint32_t unit = 0;
            for (uint32_t nrun = 0; read_run(nrun); ++nrun) {
                const int32_t all_see = s.len + s.token0;  // the last key that all rows see
                for (int32_t k = 0; ok && k < s.n; ++k, ++unit) {
                    const uint32_t st = (2 * unit + 1) % N;
                    ok = tc_wait_warp(&full[1][unit % kReady], (unit / kReady) & 1);
                    if (!ok) break;
                    const int32_t key0 = (s.first + k) * kUnitKeys;
                    const uint4 there = *reinterpret_cast<const uint4 *>(s_exist[unit % kReady]);
                    if (key0 + kUnitKeys > all_see + 1 || (there.x & there.y & there.z & there.w) != 0xffffffffu) {
                        bool found = false;
#pragma unroll 1
                        for (int at = lane; at < kUnitKeys; at += kWarp) {
                            uint8_t *line = sm_kv + st * S::kTile + at * 128;
                            const bool gone = !((s_exist[unit % kReady][at / 32] >> (at & 31)) & 1);
                            if (!gone && key0 + at <= all_see) continue;
#pragma unroll 1
                            for (int c = 0; c < D / 8; ++c) {  // (in an order that spreads the lanes over the banks)
                                uint4 *piece = reinterpret_cast<uint4 *>(line + (c / 8) * kBlock16 + ((c ^ at) & 7) * 16);
                                uint4 v = make_uint4(0, 0, 0, 0);
                                if (!gone) {
                                    v = *piece;
                                    uint32_t *w[4] = {&v.x, &v.y, &v.z, &v.w};
                                    constexpr uint32_t kMax = F16 ? 0x7c00u : 0x7f80u;
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        uint32_t keep = 0xffffffffu;
                                        if ((*w[e] & kMax) == kMax) keep &= 0xffff0000u;
                                        if ((*w[e] >> 16 & kMax) == kMax) keep &= 0x0000ffffu;
                                        found |= keep != 0xffffffffu;
                                        *w[e] &= keep;
                                    }
                                }
                                *piece = v;
                            }
                        }
                        if (found) s_cleared[nrun % kRuns] = nrun + 1;
                        fence_proxy_async();
                    }
                    warp_arrive(&ready[unit % kReady]);
                }
            }
        } else {
            // --------------------------------------------------------------------------------------- runs, and their queries
            uint32_t qx = 0;
            for (uint32_t nrun = 0;; ++nrun) {
                const bool more = ok && runs.next(a, s);
                if (lane == 0) {
                    s_run[nrun % kRuns][0] = make_int4(s.b, s.hk, s.rt, s.part);
                    s_run[nrun % kRuns][1] = make_int4(s.len, s.token0, s.tokens, s.keys);
                    s_run[nrun % kRuns][2] = make_int4(s.first, more ? s.n : 0, s.units, s.parts);
                    mbar_arrive(&run_full[nrun % kRuns]);
                }
                if (!more) break;
                const int rows = s.tokens * a.group;
                const uint32_t q0 = qx, end = qx + (rows <= kSlotRows ? 1 : 2);
                constexpr int kVec = D / 8, kStep = kWarp / kVec;  // vectors of a row, rows of a pass
                const int c = lane % kVec, in_pass = lane / kVec;
                int g = in_pass % a.group;  // (a row's query head in its key head's)
                const uint16_t *q = a.q + s.b * a.qs[0] + (s.token0 + in_pass / a.group) * a.qs[1] + (int64_t(s.hk) * a.group + g) * a.qs[2] + 8 * c;
                const int64_t next = kStep * a.qs[2], wrap = a.qs[1] - a.group * a.qs[2];
                for (int row0 = 0; qx < end; ++qx, row0 += kSlotRows) {
                    if (qx >= NQ) ok = ok && tc_wait_warp(&q_free[qx % NQ], (qx / NQ - 1) & 1);
                    if (!ok) break;
                    const int last = min(rows - row0, kSlotRows);
                    uint8_t *dst = sm_q + (qx % NQ) * S::kQ + (c / 8) * kBlock16 + in_pass * 128;
#pragma unroll 1
                    for (int row = in_pass; row < last; row += kStep, dst += kStep * 128) {
                        cp_async16(dst + (((c & 7) ^ (row & 7)) * 16), q);
                        q += next;
                        for (g += kStep; g >= a.group; g -= a.group) q += wrap;
                    }
                    cp_async_commit();
                }
                for (uint32_t x = q0; x < qx; ++x) {
                    if (x + 1 < qx)
                        cp_async_wait<1>();
                    else
                        cp_async_wait<0>();
                    fence_proxy_async();
                    warp_arrive(&q_ready[x % NQ]);
                }
            }
            fill_absent(a, cta, gridDim.x);  // (the others are still at the last runs)
        }
    }
    if (!ok) s_bad = 1;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kMmaWarp16)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(kColumns16) : "memory");
    // (the thread that wrote it last; the join writes the statuses)
    if (s_bad && tid == kFirstSlotWarp * kWarp) a.desc[2 * cta].w |= kLate;
}

// Joins the partial results of the items that several CTAs hold, and writes the statuses of a launch that a CTA gave up: CTAs
// (i, .) look after the item whose first part is the i-th CTA's, a warp a query row, adding the parts in order, kJoinFlight on
// their way together.  (4 / 6 / 8 / 12, then: 13.8 / 13.0 / 13.2 / 14.2 us for one token over 2K, 115.4 / 113.0 / 115.8 / 117.2 for
// chunks of 500 tokens.)
constexpr int kJoinWarps16 = 8, kJoinFlight = 6;
template <bool F16, int D>
__global__ void __launch_bounds__(kJoinWarps16 *kWarp, 3) attn16_join_kernel(const Attn16Args a) {
    constexpr int E = D / kWarp;  // dimensions of a lane
    using Part = typename std::conditional<E == 4, float4, float2>::type;
    const int i = blockIdx.x, lane = threadIdx.x & 31, warp = int(blockIdx.y) * kJoinWarps16 + (threadIdx.x >> 5), warps = int(gridDim.y) * kJoinWarps16;
    pdl_wait();
    pdl_trigger();
    // the item's first part is the CTA's second partial result, or its first one
    const int4 first = __ldcg(a.desc + 2 * i), second = __ldcg(a.desc + 2 * i + 1);
    if ((first.w & kLate) && blockIdx.y == 0 && a.status)
        // some row is not done; which ones, the CTA does not know
        for (int b = threadIdx.x; b < a.B; b += kJoinWarps16 * kWarp) a.status[b] = SWITCHSD_ROW_TIMEOUT;
    const bool is_second = second.x >= 0 && (second.w & kFirst);
    const int4 de = is_second ? second : first;
    if (de.x >= 0 && (de.w & kFirst)) {
        const int n = de.w >> 16, rows = (de.w >> 3) & 0x1fff, from = 2 * i + is_second;
        for (int row = warp; row < rows; row += warps) {
            float mx = kFloor, sum = 0.f, y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = 0.f;
            for (int j0 = 0; j0 < n; j0 += kJoinFlight) {
                float pm[kJoinFlight], ps[kJoinFlight], top = mx;
                Part py[kJoinFlight];
#pragma unroll
                for (int j = 0; j < kJoinFlight; ++j) {
                    pm[j] = kFloor;
                    ps[j] = 0.f;
                    py[j] = Part{};
                    if (j0 + j < n) {
                        const float *src = a.part + (size_t(j0 + j ? 2 * (i + j0 + j) : from) * kTileRows + row) * (D + kPartExtra);
                        const float2 ms = __ldcg(reinterpret_cast<const float2 *>(src + D));
                        pm[j] = ms.x;
                        ps[j] = ms.y;
                        py[j] = __ldcg(reinterpret_cast<const Part *>(src) + lane);
                    }
                }
#pragma unroll
                for (int j = 0; j < kJoinFlight; ++j) top = fmaxf(top, pm[j]);
                const float f0 = exp2_approx(mx - top);
                sum *= f0;
#pragma unroll
                for (int e = 0; e < E; ++e) y[e] *= f0;
#pragma unroll
                for (int j = 0; j < kJoinFlight; ++j) {
                    const float f = exp2_approx(pm[j] - top);
                    sum = fmaf(ps[j], f, sum);
                    const float *p = reinterpret_cast<const float *>(&py[j]);
#pragma unroll
                    for (int e = 0; e < E; ++e) y[e] = fmaf(p[e], f, y[e]);
                }
                mx = top;
            }
            const int t = de.z + row / a.group, h = de.y * a.group + row % a.group;
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            uint32_t *out = reinterpret_cast<uint32_t *>(a.out + ((size_t(de.x) * a.T + t) * a.Hq + h) * D) + lane * (E / 2);
            if constexpr (E == 4)
                *reinterpret_cast<uint2 *>(out) = make_uint2(narrow2<F16>(y[0] * inv, y[1] * inv), narrow2<F16>(y[2] * inv, y[3] * inv));
            else
                *out = narrow2<F16>(y[0] * inv, y[1] * inv);
        }
    }
}

// Whether the environment variable SWITCHSD_DIAG_ATTENTION_GIVE_UP is 1 (read once per process): a diagnostic of the path
// behind a wait that ran out.  The warp of the products issues none and waits for nothing, so the others' waits run out, the query
// rows' in every CTA that has a run: what the statuses then say comes from them.
static bool give_up16() {
    static const bool set = [] {
        const char *v = std::getenv("SWITCHSD_DIAG_ATTENTION_GIVE_UP");
        return v != nullptr && v[0] == '1' && v[1] == '\0';
    }();
    return set;
}

static size_t workspace16(int D) { return size_t(2 * kMaxCtas16) * (sizeof(int4) + size_t(kTileRows) * (D + kPartExtra) * sizeof(float)) + 32; }

// The cache as [pages][2 Hkv][page][D], a box of 64 dimensions of the tokens of a unit that lie in one page.
static bool encode_cache(CUtensorMap *map, const switchsd_kv16_attention_params *p) {
    PFN_cuTensorMapEncodeTiled_v12000 fn = tensor_map_encoder();
    if (fn == nullptr) return false;
    const cuuint64_t D = cuuint64_t(p->D), P = cuuint64_t(p->page), H2 = 2 * cuuint64_t(p->Hkv);
    const cuuint64_t dims[4] = {D, P, H2, cuuint64_t(p->pages)}, strides[3] = {2 * D, 2 * D * P, 2 * D * P * H2};
    const cuuint32_t box[4] = {64, cuuint32_t(std::min(kUnitKeys, int(p->page))), 1, 1}, one[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 4, const_cast<void *>(p->cache), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool F16, int D>
static cudaError_t launch16(const CUtensorMap &map, const Attn16Args &a, cudaStream_t s) {
    static bool attr_done[64] = {false};
    const int sms = sm_count();
    int dev = 0;
    cudaError_t e = sms ? cudaGetDevice(&dev) : cudaErrorInvalidDevice;
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_done[dev]) {
        e = cudaFuncSetAttribute(attn16_kernel<F16, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem16<D>::bytes);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_done[dev] = true;
    }
    const unsigned ctas = unsigned(std::min(kMaxCtas16, sms));
    // an explicit one-CTA cluster: the MMA commit addresses shared::cluster
    e = launch_pdl(attn16_kernel<F16, D>, dim3(ctas), dim3(kThreads16), size_t(Smem16<D>::bytes), s, 1u, map, a);
    if (e != cudaSuccess) return e;
    // (two waves of CTAs at the most)
    const int64_t rows = std::min(int64_t(a.tokens), int64_t(a.T)) * a.group;
    return launch_pdl(attn16_join_kernel<F16, D>, dim3(ctas, unsigned(std::min(int64_t(6), (rows + kJoinWarps16 - 1) / kJoinWarps16))), dim3(kJoinWarps16 * kWarp), 0, s, 0u, a);
}

}  // namespace switchsd

using namespace switchsd;

extern "C" size_t switchsd_kv16_attention_workspace_bytes(const switchsd_kv16_attention_params *p) {
    return p && kv4_dim_ok(p->D) ? workspace16(p->D) : 0;
}

extern "C" int switchsd_kv16_attention(const switchsd_kv16_attention_params *p) {
    if (!p || !p->q || !p->cache || !p->block_table || !p->lens || !p->new_lens || !p->out || !p->workspace) return SWITCHSD_ERR_ARG;
    if (p->dtype != SWITCHSD_BF16 && p->dtype != SWITCHSD_F16) return SWITCHSD_ERR_ARG;
    if (!aligned16(p->q) || !aligned16(p->cache) || !aligned16(p->out) || !aligned16(p->workspace)) return SWITCHSD_ERR_ARG;
    const int32_t sizes[3] = {p->B, p->T, p->Hq};
    for (int i = 0; i < 3; ++i)
        if (!stride_ok(p->q_stride[i], sizes[i])) return SWITCHSD_ERR_ARG;
    if (p->B < 1 || p->T < 1 || p->Hq < 1 || p->Hkv < 1 || p->Hq % p->Hkv != 0 || p->Hq / p->Hkv > 64 || p->blocks < 1 || p->pages < 1 ||
        !kv4_page_ok(p->page) || !kv4_dim_ok(p->D))
        return SWITCHSD_ERR_SHAPE;
    if (int64_t(p->pages) * p->page > 0x7fffffff || int64_t(p->blocks) * p->page > 0x7fffffff - 1024 || int64_t(p->B) * p->T > 0x7fffffff ||
        int64_t(p->T) * (p->Hq / p->Hkv) > 0x7fffffff)
        return SWITCHSD_ERR_SHAPE;
    if (p->workspace_bytes < switchsd_kv16_attention_workspace_bytes(p)) return SWITCHSD_ERR_ARG;
    Attn16Args a = {};
    a.q = static_cast<const uint16_t *>(p->q);
    for (int i = 0; i < 3; ++i) a.qs[i] = stride_of(p->q_stride[i], sizes[i]);
    a.cache = static_cast<const uint8_t *>(p->cache);
    a.table = p->block_table;
    a.lens = p->lens;
    a.new_lens = p->new_lens;
    a.out = static_cast<uint16_t *>(p->out);
    a.status = p->status;
    a.desc = static_cast<int4 *>(p->workspace);
    a.part = reinterpret_cast<float *>((reinterpret_cast<uintptr_t>(a.desc + 2 * kMaxCtas16) + 31) & ~uintptr_t(31));
    a.B = p->B;
    a.T = p->T;
    a.Hq = p->Hq;
    a.Hkv = p->Hkv;
    a.pages = p->pages;
    a.blocks = p->blocks;
    a.page_shift = log2_of(p->page);
    a.lens_add = p->lens_add;
    a.new_add = p->new_add;
    a.group = p->Hq / p->Hkv;
    a.dim = p->D;
    a.scale = p->scale;
    a.give_up = give_up16();
    a.tokens = kTileRows / a.group;
    CUtensorMap map;
    if (!encode_cache(&map, p)) return SWITCHSD_ERR_CUDA;
    cudaStream_t s = static_cast<cudaStream_t>(p->stream);
    cudaError_t e;
    if (p->dtype == SWITCHSD_F16)
        e = p->D == 128 ? launch16<true, 128>(map, a, s) : launch16<true, 64>(map, a, s);
    else
        e = p->D == 128 ? launch16<false, 128>(map, a, s) : launch16<false, 64>(map, a, s);
    return e == cudaSuccess ? SWITCHSD_OK : SWITCHSD_ERR_CUDA;
}
