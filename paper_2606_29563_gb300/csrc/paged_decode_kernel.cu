// Attention of one new token per sequence over the paged cache, with an optional sliding
// window and first slots that stay visible:
//   out = sum_j p_j v_j,  p_j = 2^(x_j - m) / sum_i 2^(x_i - m),  x_j = scale log2(e) <q, k_j>,
// and weights[slot j] += the sum of p_j over the query heads of the KV head.
//
// Every visible row of K and V is read once; a KV head's query heads share it.  A warp
// works alone on blocks of 16 slots (of one page): a lane brings the block's four tiles of
// 16 rows x 64 columns by TMA (128-byte swizzle) into the warp's ring, logits and weighted
// values are m16n8k16 tiles (tcgen05 tiles of 64 rows and more would leave the up to eight
// query heads most of the tile empty).  For the values the tile's upper eight rows hold the
// heads' weights rounded to the cache's type and the lower eight what the rounding left, so
// that the weights count with 16 bits and more at no further instruction.
//
// The work is the list of all blocks of all (sequence, KV head) pairs in order, which the
// CTAs share evenly: the lengths are on the device, and no grid over sequences fits a long
// and a short one.  A pair that lies in one CTA's share is finished there; the shares of a
// pair that several have meet in paged_join_kernel, in the order of the shares.  The weights
// need a row's final sums: the logits wait for them in scratch (4 bytes a query head and
// slot beside 512 of keys and values).
//
// With few pairs the CTAs of a pair form a cluster, and with short ones each has a CTA; these
// meet over distributed shared memory in one launch.
//
// HBM-bound when there is much to read: 131072 slots of 8 heads (537 MB) in 86 us, 6.3 TB/s, 92 %
// of the measured copy rate; 64 rows of 1024 to 2048 slots of 4 heads and 7 query heads each (203 MB
// with the weights) in 48 us, of which the reading takes 31: before it lie the lengths, the
// list, the pages' numbers and the first copies (4 us), behind it the merge, the weights (7 us, each
// round a chain of loads) and an empty join.  512 slots 6.2 us, the same chain once.  The join's grid goes
// by the bound on the lengths: the 64 rows take 51 us under one of 8192, 57 of 32768 and 82 of 131072.
//
// Rows of 8 bits (E8): blocks of 32 slots, whose numbers a warp turns into fp16 for the same tiles.  131072 slots of 8 heads (277
// MB) in 53 us, 5.2 TB/s; the 64 rows above (107 MB) in 38.3 us; 512 slots 7.6.  A block takes a warp 1.6 us, 3000 cycles for 8.4
// KB: eight warps on each of 148 SMs read at the copy rate (304 equal pairs: 6.7 to 7.1 TB/s for each slot more).  What lies
// above the floor is the start (6.5 us of the 131072 slots) and the join (3), and of the 64 rows the pairs' lengths: the
// longest CTA's warps have 16 blocks, 10.4 would be even.  A third of a block's cycles are the conversions (128 of two numbers
// each, two cycles of a scheduler).  What that took, 131072 slots and the 64 rows: blocks of 16 slots 72 and 49;
// eight warps of 128 registers a CTA 73 and 42; 32 slots, the logits as tiles of e4m3 57 and 46; as tiles of fp16, copies
// issued before a block is worked on 54 and 39.5; the rows of 32 loads found at once 52.6 and 37.6 (a head's power of two by
// its products, where a warp's scales alone had lost small values beside a large one without weight: 52.9 and 38.3).
// Slower: three CTAs an SM with rings of two blocks (61 and 42).
//
// Behind prefixes that groups of sequences share (OPEN): a sequence's own slots as above, then the prefixes as tiles of the prefill
// kernel (prefill_kernel.cu), whose CTAs begin where this kernel's end, and one join of all their sums.  160 sequences
// of 1 to 1000 slots (328 MB) in three groups of 101, 42 and 17 behind 32768, 8001 and 20000 (249 MB), 8 heads, in 140 us: the own
// slots 60, the prefixes 75 more, the join 5 (own slots of 8 bits 132 in all); 64 of 16 to 527 behind 4096 34 us (12, 15 and 8);
// 4 behind 500 14 us (4, 7 and 3), three launches' chains of loads.
#include "half_types.cuh"
#include "kvec_internal.cuh"
#include "prefix_list.cuh"
#include "sm100_ptx.cuh"

#include <cooperative_groups.h>

#include <algorithm>
#include <type_traits>

namespace kvec {

namespace {

namespace cg = cooperative_groups;

constexpr int kPdWarps = 4;
constexpr int kPdThreads = 32 * kPdWarps;
constexpr int kPdStages = 3;                 // blocks in a warp's ring
constexpr int kPdHalf = 16;                  // slots that are surely of one page
// Slots of a block: with 8 bits two halves of 16, each with a page of its own.
template <bool E8>
constexpr int kPdBlock = E8 ? 32 : 16;
constexpr int kPdTile = 16 * 128;            // bytes of 16 rows x 64 columns, or of 16 whole rows of 8 bits
constexpr int kPdStage = 4 * kPdTile;        // K columns 0-63, 64-127, V the same; 8 bits: 32 rows of K, of V
constexpr int kPdSmem = kPdWarps * kPdStages * kPdStage + 1024;
constexpr int kPdCtasPerSm = 2;
constexpr int kPdMaxCluster = 8;
constexpr int kPdHeads = 8;                  // most query heads of a KV head
constexpr int kPairCost = 12;                // what beginning and ending a pair takes, in blocks
constexpr int kJoinThreads = 128;
constexpr int kJoinRows = 8 * kJoinThreads;  // slots of a join block's weights, two times four a thread
// The maximum before the first logit: the lowest finite value, so that a logit of minus
// infinity gets the weight 2^-inf = 0 there too, and not 2^(-inf + inf).
constexpr float kNoLogit = -3.402823466e38f;

struct PdArgs {
    CUtensorMap kmap, vmap;   // [rows][128], boxes of 16 x 64; 8 bits: of 16 or 32 rows of 128 bytes
    PagedCacheView c;
    PagedDecodeIO io;
    float* logits;            // [pair][nbmax][g][slots of a block]
    float* part_o;            // [2 * ctas][8][128] shares of split pairs, unnormalised
    float2* part_ml;          // [2 * ctas][8] their maxima and sums
    float* own_o;             // shared_decode: [pair][g][128] sums of whole pairs, in the rows behind part_o's, and
    float2* own_ml;           // [pair][g] behind part_ml's; then come the prefixes'
    longlong2* own_plan;      // [batch] (places before the sequence, -), and (all places, whether each pair is a CTA's)
    const PrefixPlan* prefix_plan;   // [batch]
    int ctas;                 // that share the list of blocks
    int pairs;                // batch * Hkv where a CTA each may do, else 0
    int nbmax;                // most visible blocks of a pair
    int g;
    int box;                  // 8 bits: rows of a copy, 32 where pages have that many
    float sl2;                // scale * log2(e)
    int fault;                // test of the error path (kvec_set_test_fault): warp 0 of CTA 0 loads nothing
};

// A sequence's visible slots and the blocks that hold them: blocks 0 .. first - 1, then
// from block `from` on.
template <int B>
struct Visible {
    int n, lo, sinks;     // slots [0, min(sinks, n)) and [lo, n)
    int first, from, nb;
    __device__ __forceinline__ void init(const PdArgs& A, int s) {
        n = min(max(__ldg(&A.c.lens[s]), 0), A.io.max_len);
        lo = A.io.window ? max(n - A.io.window, 0) : 0;
        sinks = min(A.io.sinks, lo);
        first = (sinks + B - 1) / B;
        from = lo / B;
        if (first >= from) first = from = 0;
        nb = first + (n + B - 1) / B - from;
    }
    __device__ __forceinline__ int block(int i) const { return i < first ? i : from + i - first; }
    __device__ __forceinline__ bool sees(int slot) const { return slot < n && (slot >= lo || slot < sinks); }
    __device__ __forceinline__ bool whole(int b) const {
        return (b + 1) * B <= n && (b * B >= lo || (b + 1) * B <= sinks);
    }
};

// Row of a slot for KV head h; -1 on no page.
__device__ __forceinline__ int slot_row(const PdArgs& A, int s, int h, int slot) {
    const int page = __ldg(&A.c.table[(size_t)s * A.c.max_pages + (slot >> A.c.log_page)]);
    if (page < 0 || page >= A.c.num_pages) return -1;
    return (int)((((unsigned)page * (unsigned)A.io.Hkv + (unsigned)h) << A.c.log_page) +
                 (unsigned)(slot & ((1 << A.c.log_page) - 1)));
}
// A block's first rows, -1 where there is none: of its 16 slots, or of two halves, of which the second may lie behind the bound
// and the table.
template <int B>
using BlockRows = std::conditional_t<(B > kPdHalf), int2, int>;
template <int B>
__device__ __forceinline__ BlockRows<B> no_rows() {
    if constexpr (B > kPdHalf) return make_int2(-1, -1);
    else return -1;
}
template <int B>
__device__ __forceinline__ BlockRows<B> block_rows(const PdArgs& A, int s, int h, int b) {
    const int first = slot_row(A, s, h, b * B);
    if constexpr (B > kPdHalf) {
        const int slot = b * B + kPdHalf;
        if (A.box == B) return make_int2(first, first < 0 ? -1 : first + kPdHalf);
        return make_int2(first, slot < A.io.max_len ? slot_row(A, s, h, slot) : -1);
    } else {
        return first;
    }
}

// A place in the list of blocks: block i of pair (s, h).
template <int B>
struct Walker {
    int s, h, i;
    Visible<B> v;
    __device__ __forceinline__ void advance(const PdArgs& A, int by) {
        i += by;
        while (i >= v.nb && s < A.io.batch) {
            i -= v.nb;
            if (++h == A.io.Hkv) {
                h = 0;
                if (++s < A.io.batch) v.init(A, s);
            }
        }
    }
};

// The list of all blocks as a warp sees it: lane l holds those of the sequences l * per .. l *
// per + per - 1, over all KV heads.  Ahead of a pair's blocks stand kPairCost places without one,
// so that a share of many short pairs does not take longer than others (32 rows of 100 to 4000
// slots 75 us without, 68 with 4, 60 with 8, 56 with 12 and 16, 58 with 28).
template <int B>
struct List {
    int per, longest;                // most blocks of a pair
    int pairs_before, pairs;         // with blocks: of the lanes before, of all
    long long before, mine, total;   // places: of the lanes before, of this lane, of all
    __device__ __forceinline__ static int places(const Visible<B>& v) { return v.nb ? v.nb + kPairCost : 0; }
    __device__ __forceinline__ void init(const PdArgs& A) {
        const int lane = threadIdx.x & 31;
        per = (A.io.batch + 31) >> 5;
        mine = 0;
        int most = 0, own = 0;
        for (int k = 0; k < per; ++k) {
            const int s = lane * per + k;
            if (s >= A.io.batch) break;
            Visible<B> v;
            v.init(A, s);
            mine += places(v);
            own += v.nb ? A.io.Hkv : 0;
            most = max(most, v.nb);
        }
        longest = __reduce_max_sync(0xffffffffu, most);
        mine *= A.io.Hkv;
        long long upto = mine;
        int upto_pairs = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, upto, o);
            const int z = __shfl_up_sync(0xffffffffu, upto_pairs, o);
            if (lane >= o) {
                upto += y;
                upto_pairs += z;
            }
        }
        before = upto - mine;
        pairs_before = upto_pairs - own;
        total = __shfl_sync(0xffffffffu, upto, 31);
        pairs = __shfl_sync(0xffffffffu, upto_pairs, 31);
    }
    // Whether each pair is a CTA's.  That saves the join, but the longest pair must not hold up the others: a
    // block takes a CTA alone 0.25 us, all places together take 0.0013 us each, and the join and the shares'
    // ends about 5 us.  Measured, by pair and by share: 64 rows of 1024 to 2048 slots 48 and 54, 64 of
    // 200 to 3200 65 and 54, 30 of 100 to 3100 58 and 44, one of 8000 beside 31 of 500 129 and 28.
    // 8 bits (32 slots a block): 0.43 and 0.0014 us; 64 rows of 1024 to 2048 37.9 and 39.4, 32 of 100 to 4000 50 and 39.
    __device__ __forceinline__ bool whole_pairs(const PdArgs& A) const {
        if constexpr (B == kPdBlock<true>) return A.pairs && (long long)longest * 300 <= total + 14 * 300;
        return A.pairs && (long long)longest * 190 <= total + 20 * 190;
    }
    // The first block from place `at` on; returns how many are before it.
    __device__ __forceinline__ long long seek(const PdArgs& A, long long at, Walker<B>& w) const {
        const uint32_t past = __ballot_sync(0xffffffffu, at < before + mine);
        w.s = A.io.batch;
        w.h = w.i = 0;
        w.v.nb = 0;
        if (!past) return total - (long long)pairs * kPairCost;
        const int l = __ffs(past) - 1;
        const long long whole = at;
        at -= __shfl_sync(0xffffffffu, before, l);
        int p = __shfl_sync(0xffffffffu, pairs_before, l);
        for (w.s = l * per;; ++w.s) {
            w.v.init(A, w.s);
            const long long here = (long long)places(w.v) * A.io.Hkv;
            if (at < here) break;
            at -= here;
            p += here ? A.io.Hkv : 0;
        }
        w.h = (int)at / places(w.v);          // at < 2^22
        const int i = (int)at - w.h * places(w.v);
        w.i = max(i - kPairCost, 0);
        return whole - (long long)(p + w.h) * kPairCost - min(i, kPairCost);
    }
    // Places of the sequences before s, by a whole warp.
    __device__ __forceinline__ long long places_before(const PdArgs& A, int s) const {
        const int l = s / per;
        return __shfl_sync(0xffffffffu, before, l) + sum_by_lanes(l * per, s, [&](int k) {
                   Visible<B> v;
                   v.init(A, k);
                   return (long long)places(v) * A.io.Hkv;
               });
    }
};

// a / b, in 32 bits where they do.
__device__ __forceinline__ long long quotient(long long a, long long b) {
    return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}
__device__ __forceinline__ long long share_start(long long total, int cta, int ctas) { return quotient(total * cta, ctas); }

__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}

// The power of two that brings a magnitude to [2^E, 2^(E + 1)), within the range of normal numbers on both sides, and its
// inverse.  In fp16's range (E = 14) products lose nothing near their largest factor then, and 2^-39 of it at most.
template <int E>
__device__ __forceinline__ float to_range(float a) {
    return __uint_as_float((uint32_t)min(254 + E - (int)(__float_as_uint(a) >> 23), 253) << 23);
}
__device__ __forceinline__ float inverse_power(float p) { return __uint_as_float((254u << 23) - __float_as_uint(p)); }
// a / b of two such, within the range of normal numbers.
__device__ __forceinline__ float power_ratio(float a, float b) {
    return __uint_as_float((uint32_t)min(max(127 + (int)(__float_as_uint(a) >> 23) - (int)(__float_as_uint(b) >> 23), 1), 254) << 23);
}

// The products with the weights' roundings and with what these left.  Against an infinite value the rest, which is
// zero or has either sign, would make NaN of what the roundings give alone.
__device__ __forceinline__ float with_rest(float hi, float lo) { return fabsf(hi) < INFINITY ? hi + lo : hi; }

// The attention weights of four slots of a block: what is read for them, and their sum over
// the query heads once these' (maximum, 1 / sum) are known.
template <int B>
struct SlotWeights {
    float4 x[kPdHeads], w;
    int row;          // of the first, -1: none of them is visible or they are on no page
    bool seen[4];
    // The e-th four slots of the pair's blocks from block i0 on.
    __device__ __forceinline__ void load(const PdArgs& A, int s, int h, const Visible<B>& v, int i0, int e) {
        const int i = i0 + e / (B / 4), r = e % (B / 4) * 4, slot = v.block(i) * B + r;
        row = slot < A.io.max_len ? slot_row(A, s, h, slot) : -1;   // past the bound the table may end
        bool any = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) any |= seen[k] = v.sees(slot + k);
        row = any ? row : -1;
        if (row < 0) return;
        const float* lg = A.logits + (((size_t)s * A.io.Hkv + h) * A.nbmax + i) * (size_t)(A.g * B) + r;
#pragma unroll
        for (int j = 0; j < kPdHeads; ++j)
            if (j < A.g) x[j] = *reinterpret_cast<const float4*>(lg + j * B);
        w = *reinterpret_cast<const float4*>(A.c.weights + row);
    }
    __device__ __forceinline__ void store(const PdArgs& A, const float* mx, const float* inv) const {
        if (row < 0) return;
        float p[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < kPdHeads; ++j) {
            if (j >= A.g) break;
            const float m = mx[j], f = inv[j];
            p[0] = fmaf(ptx::ex2(x[j].x - m), f, p[0]);
            p[1] = fmaf(ptx::ex2(x[j].y - m), f, p[1]);
            p[2] = fmaf(ptx::ex2(x[j].z - m), f, p[2]);
            p[3] = fmaf(ptx::ex2(x[j].w - m), f, p[3]);
        }
        *reinterpret_cast<float4*>(A.c.weights + row) =
            make_float4(seen[0] ? w.x + p[0] : w.x, seen[1] ? w.y + p[1] : w.y, seen[2] ? w.z + p[2] : w.z,
                        seen[3] ? w.w + p[3] : w.w);
    }
};

// Adds the attention weights of blocks [i0, i1) of pair (s, h) to the cache's.  One quarter of
// a thread's at a time: two at once take 36 registers more in the decode kernel, which spills
// then, and 40 in the join, of which fewer blocks are resident (64 rows of 1024 to 2048 slots
// 59.6 us, 54.3 with one; a thread a slot 78).
template <int NT, int B>
__device__ void add_weights(const PdArgs& A, int s, int h, const Visible<B>& v, int i0, int i1, const float* mx,
                            const float* inv) {
    const int n = (i1 - i0) * (B / 4);
#pragma unroll 1
    for (int e = threadIdx.x; e < n; e += NT) {
        SlotWeights<B> a;
        a.load(A, s, h, v, i0, e);
        a.store(A, mx, inv);
    }
}

// CL: a cluster of CTAs per pair (grid splits x Hkv x batch) instead of a share of the list.
// E8: rows of e4m3 numbers with a scale each, which multiplies a key's logit and a value's weight.  The numbers become fp16,
// which holds them all, on their way from shared memory to the tiles; queries of bf16 and the weights with their
// scales are brought to its range by powers of two, a row's and that of a head's largest product so far.  (Tiles of e4m3, m16n8k32, with a
// query as the sum of two or three numbers took more: their operands are converted too, the queries every time.)
// OPEN: pairs' sums stay sums (own_o, own_ml), for shared_join_kernel, which adds the weights too.
template <class T, bool CL, bool E8, bool OPEN>
__global__ void __launch_bounds__(kPdThreads, kPdCtasPerSm) paged_decode_kernel(const __grid_constant__ PdArgs A) {
    constexpr int B = kPdBlock<E8>;
    constexpr bool kEarly = E8 || OPEN;                         // two blocks in flight beside the one that is worked on
    using Operand = std::conditional_t<E8, __half, T>;          // the tiles' type
    extern __shared__ uint8_t pd_smem_raw[];
    // 1024-byte alignment for the swizzled tiles.
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(pd_smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ __align__(8) uint64_t full[kPdWarps][kPdStages];
    __shared__ BlockRows<B> srow[kPdWarps][kPdStages];          // the staged block's
    __shared__ __align__(16) float scales[kPdWarps][E8 ? kPdStages : 1][2][B];   // of the staged block's K and V
    __shared__ float wm[kPdWarps][kPdHeads], wl[kPdWarps][kPdHeads];
    __shared__ float* wacc[kPdWarps];                           // the warps' outputs, each in its free stage
    __shared__ float cm[kPdHeads], cl[kPdHeads], fm[kPdHeads], finv[kPdHeads];
    __shared__ __align__(16) float co[CL ? kPdHeads : 1][kHeadDim];
    const int tid = threadIdx.x, lane = tid & 31, warp = ptx::warp_uniform(tid >> 5);
    const int Hq = A.io.Hq, Hkv = A.io.Hkv, g = A.g;
    if (tid == 0) {
        ptx::prefetch_tensormap(&A.kmap);
        ptx::prefetch_tensormap(&A.vmap);
        for (int w = 0; w < kPdWarps; ++w)
            for (int i = 0; i < kPdStages; ++i) ptx::mbar_init(&full[w][i], 1);
        ptx::fence_barrier_init();
    }
    __syncthreads();
    // The trigger follows the wait: what was complete before this grid may be read by the
    // join kernel before its own wait.
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");

    // This CTA's blocks: `count` from (s, h, i) on.
    Walker<B> cur;
    int count;   // a share of at most 65535 * 32 * 2^16 blocks
    int splits = 1, rank = 0;
    if constexpr (CL) {
        splits = (int)gridDim.x;
        rank = (int)blockIdx.x;
        cur.s = blockIdx.z;
        cur.h = blockIdx.y;
        cur.v.init(A, cur.s);
        cur.i = cur.v.nb * rank / splits;
        count = cur.v.nb * (rank + 1) / splits - cur.i;
    } else {
        List<B> list;
        list.init(A);
        if constexpr (OPEN) {   // for the join, which would take as long for each block to find them
            if (warp == 1)
                for (int s = blockIdx.x; s < A.io.batch; s += A.ctas) {
                    const long long at = list.places_before(A, s);
                    if (lane == 0) A.own_plan[s] = make_longlong2(at, 0);
                }
            if (blockIdx.x == 0 && tid == 0) A.own_plan[A.io.batch] = make_longlong2(list.total, list.whole_pairs(A) ? 1 : 0);
        }
        if (list.whole_pairs(A)) {
            cur.s = blockIdx.x / Hkv;
            cur.h = blockIdx.x - cur.s * Hkv;
            cur.i = cur.v.nb = 0;
            if ((int)blockIdx.x < A.pairs) cur.v.init(A, cur.s);
            count = cur.v.nb;
        } else {
            const long long first = list.seek(A, share_start(list.total, blockIdx.x, A.ctas), cur);
            Walker<B> end;
            count = (int)(list.seek(A, share_start(list.total, blockIdx.x + 1, A.ctas), end) - first);
        }
    }

    uint8_t* ring = smem + warp * (kPdStages * kPdStage);
    const uint32_t ring32 = ptx::smem_u32(ring);
    // Loads: this warp's blocks are warp, warp + 4, ... of the CTA's; load number k goes to
    // stage k % kPdStages, and one stage is free while a block is worked on.
    // The rows of the next two are fetched ahead: a page's number takes as long as its rows.  kEarly: those of 32 at
    // once, a lane each.
    Walker<B> ld = cur;
    int ld_at = warp, row_at = warp;      // the next load, the next row to fetch
    if (row_at < count) ld.advance(A, warp);
    BlockRows<B> ahead = no_rows<B>();    // kEarly: of the load lane loads on from the last fetch
    int taken = 32;
    auto next_row = [&]() {
        if constexpr (kEarly) {
            if (taken == 32) {
                taken = 0;
                const int mine = row_at + lane * kPdWarps;
                ahead = no_rows<B>();
                if (mine < count) {
                    Walker<B> w = ld;
                    w.advance(A, lane * kPdWarps);
                    ahead = block_rows<B>(A, w.s, w.h, w.v.block(w.i));
                }
                row_at += 32 * kPdWarps;
                if (row_at < count) ld.advance(A, 32 * kPdWarps);
                __syncwarp();
            }
            BlockRows<B> row;
            if constexpr (E8) row = make_int2(__shfl_sync(0xffffffffu, ahead.x, taken), __shfl_sync(0xffffffffu, ahead.y, taken));
            else row = __shfl_sync(0xffffffffu, ahead, taken);
            ++taken;
            return row;
        } else {
            if (row_at >= count) return no_rows<B>();
            const BlockRows<B> row = block_rows<B>(A, ld.s, ld.h, ld.v.block(ld.i));
            row_at += kPdWarps;
            if (row_at < count) ld.advance(A, kPdWarps);
            return row;
        }
    };
    BlockRows<B> rows[2];
    if constexpr (!kEarly) {
        rows[0] = next_row();
        rows[1] = next_row();
    }
    int ld_stage = 0;
    bool failed = false;      // a wait gave up: no further loads and waits, outputs are invalid
    auto load_next = [&]() {
        if (ld_at < count && !failed) {
            // Warp-uniform operands: else each TMA instruction moves its own to uniform registers.
            if constexpr (kEarly) rows[0] = next_row();
            const int at = ptx::warp_uniform(ld_stage);
            if constexpr (E8) {
                const int row = ptx::warp_uniform(rows[0].x), upper = ptx::warp_uniform(rows[0].y);
                if (ptx::elect_one()) {
                    srow[warp][at] = make_int2(row, upper);
                    if ((row >= 0 || upper >= 0) && !(A.fault && warp == 0 && blockIdx.x == 0)) {
                        uint8_t* dst = ring + at * kPdStage;
                        uint64_t* bar = &full[warp][at];
                        constexpr uint32_t kHalfBytes = 2 * (kPdTile + kPdHalf * 4);
                        auto load = [&](int r, int from) {   // rows from r on, behind `from` slots of the block
                            ptx::tma_load_2d(dst + from * 128, &A.kmap, bar, 0, r);
                            ptx::tma_load_2d(dst + 2 * kPdTile + from * 128, &A.vmap, bar, 0, r);
                            ptx::bulk_load(&scales[warp][at][0][from], A.c.k_scales + r, A.box * 4, bar);
                            ptx::bulk_load(&scales[warp][at][1][from], A.c.v_scales + r, A.box * 4, bar);
                        };
                        ptx::mbar_arrive_expect_tx(bar, row >= 0 && upper >= 0 ? 2 * kHalfBytes : kHalfBytes);
                        if (row >= 0) load(row, 0);
                        if (upper >= 0 && A.box == kPdHalf) load(upper, kPdHalf);
                    }
                }
            } else {
                const int row = ptx::warp_uniform(rows[0]);
                if (ptx::elect_one()) {
                    srow[warp][at] = row;
                    if (row >= 0 && !(A.fault && warp == 0 && blockIdx.x == 0)) {
                        uint8_t* dst = ring + at * kPdStage;
                        uint64_t* bar = &full[warp][at];
                        ptx::mbar_arrive_expect_tx(bar, kPdStage);
                        ptx::tma_load_2d(dst, &A.kmap, bar, 0, row);
                        ptx::tma_load_2d(dst + kPdTile, &A.kmap, bar, 64, row);
                        ptx::tma_load_2d(dst + 2 * kPdTile, &A.vmap, bar, 0, row);
                        ptx::tma_load_2d(dst + 3 * kPdTile, &A.vmap, bar, 64, row);
                    }
                }
            }
            ld_at += kPdWarps;
            if constexpr (!kEarly) {
                rows[0] = rows[1];
                rows[1] = next_row();
            }
        }
        ld_stage = ld_stage + 1 == kPdStages ? 0 : ld_stage + 1;
    };
#pragma unroll
    for (int i = 0; i < kPdStages - 1; ++i) load_next();
    __syncwarp();

    int st = 0;               // stage of this warp's next block
    uint32_t phases = 0u;     // bit i: parity of stage i's next completion
    bool first_segment = true;
    int done = 0;             // blocks of the CTA's that precede the current segment
    while (CL || done < count) {
        // A segment: the CTA's blocks of one pair.
        const int s = cur.s, h = cur.h, i_begin = cur.i;
        const Visible<B> v = cur.v;
        const int len = min(count - done, v.nb - i_begin);
        const bool whole = len == v.nb;
        // The group's query rows as the upper half of the tile's row operand: head lane / 4.
        uint32_t qa[8][2];
        float sl2 = A.sl2;             // E8: also what the row was divided by
        if constexpr (E8) {
            // Columns 16 kk + 4 (lane % 4) and three more.
            const int j = lane >> 2;
            const uint2* qr =
                reinterpret_cast<const uint2*>(A.io.q + ((size_t)s * Hq + (size_t)h * g + (j < g ? j : 0)) * kHeadDim) + (lane & 3);
#pragma unroll
            for (int kk = 0; kk < 8; ++kk) {
                const uint2 w = j < g ? __ldg(qr + 4 * kk) : make_uint2(0u, 0u);
                qa[kk][0] = w.x;
                qa[kk][1] = w.y;
            }
            if constexpr (!std::is_same_v<T, __half>) {
                float top = 0.f;       // of the finite ones
#pragma unroll
                for (int kk = 0; kk < 16; ++kk) {
                    const float2 f = Half16<T>::unpack(qa[kk >> 1][kk & 1]);
                    top = fabsf(f.x) < INFINITY ? fmaxf(top, fabsf(f.x)) : top;
                    top = fabsf(f.y) < INFINITY ? fmaxf(top, fabsf(f.y)) : top;
                }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const float up = to_range<14>(top);
                sl2 *= inverse_power(up);
#pragma unroll
                for (int kk = 0; kk < 16; ++kk) {
                    const float2 f = Half16<T>::unpack(qa[kk >> 1][kk & 1]);
                    qa[kk >> 1][kk & 1] = Half16<__half>::pack(f.x * up, f.y * up);
                }
            }
        } else {
            const int j = lane >> 2;
            const uint32_t* qr =
                reinterpret_cast<const uint32_t*>(A.io.q + ((size_t)s * Hq + (size_t)h * g + (j < g ? j : 0)) * kHeadDim) +
                (lane & 3);
#pragma unroll
            for (int kk = 0; kk < 8; ++kk) {
                qa[kk][0] = j < g ? __ldg(qr + 8 * kk) : 0u;
                qa[kk][1] = j < g ? __ldg(qr + 8 * kk + 4) : 0u;
            }
        }
        // Head lane / 4, hi and lo.  E8: a column a head (2 (lane % 4) and the next), a row a dimension: the weights are
        // the column operand, as which their tile needs no second half, and hi and lo meet in one sum.
        constexpr int kAcc = E8 ? 8 : 16;
        float acc[kAcc][4];
#pragma unroll
        for (int d = 0; d < kAcc; ++d)
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[d][c] = 0.f;
        float m = kNoLogit, l = 0.f;   // head lane / 4; l of this lane's slots
        // E8: head lane / 4's largest weight times scale so far, relative to m; acc's columns are the sums times the power of two
        // that brings it to fp16's range.
        float peak = 0.f, up = to_range<14>(0.f);
        // The warp's first block of the segment: its blocks are warp mod kPdWarps of the CTA's.
        const int skip = (warp - done % kPdWarps + kPdWarps) % kPdWarps;
        for (int e = skip; e < len; e += kPdWarps) {
            const int i = i_begin + e, b = v.block(i);
            __syncwarp();
            if constexpr (kEarly) load_next();   // into the stage that the step before freed
            const BlockRows<B> rows_at = srow[warp][st];
            int row;                       // -1: nothing is there
            bool here[B / kPdHalf];        // by halves
            if constexpr (E8) {
                row = max(rows_at.x, rows_at.y);
                here[0] = rows_at.x >= 0;
                here[1] = rows_at.y >= 0;
            } else {
                row = rows_at;
                here[0] = row >= 0;
            }
            const uint32_t src = ring32 + st * kPdStage;
            float x[B / 8][4];
            if (row >= 0) {
                if (!failed && !__all_sync(0xffffffffu, ptx::mbar_wait(&full[warp][st], (phases >> st) & 1u))) {
                    failed = true;
                    if (lane == 0) atomicExch(A.io.err, 3);
                }
                if (!failed) phases ^= 1u << st;   // the parities stay those of copies in flight
#pragma unroll
                for (int t = 0; t < B / 8; ++t)
#pragma unroll
                    for (int c = 0; c < 4; ++c) x[t][c] = 0.f;
                if constexpr (E8) {
                    // Eight keys at a time: chunks 4 cc + lane / 8 of row lane % 8.  A lane's word holds columns 4 (lane % 4) on
                    // of a chunk: the lower two meet the tile's lower columns.
                    const int kr = lane & 7;
#pragma unroll
                    for (int cc = 0; cc < 2; ++cc)
#pragma unroll
                        for (int t = 0; t < B / 8; ++t) {
                            uint32_t kb[4];
                            ldmatrix_x4(src + (8 * t + kr) * 128 + (((4 * cc + (lane >> 3)) ^ kr) << 4), kb);
#pragma unroll
                            for (int c = 0; c < 4; ++c)
                                Half16<Operand>::mma(x[t], qa[4 * cc + c][0], 0u, qa[4 * cc + c][1], 0u, e4m3_to_half2(kb[c]),
                                                     e4m3_to_half2_upper(kb[c]));
                        }
                } else {
                    // Logits: key row (lane & 7) + 8 (lane / 16), columns 16 kk + 8 (lane / 8 % 2).
                    const int kr = (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk) {
                        uint32_t kb[4];
                        const int chunk = (2 * kk + ((lane >> 3) & 1)) & 7;
                        ldmatrix_x4(src + (kk >> 2) * kPdTile + kr * 128 + ((chunk ^ (kr & 7)) << 4), kb);
                        Half16<Operand>::mma(x[0], qa[kk][0], 0u, qa[kk][1], 0u, kb[0], kb[1]);
                        Half16<Operand>::mma(x[1], qa[kk][0], 0u, qa[kk][1], 0u, kb[2], kb[3]);
                    }
                }
            }
            // This lane's slots: 8 t + 2 (lane % 4) + c.
            const bool all = here[0] && here[B / kPdHalf - 1] && v.whole(b);
            float vs[E8 ? B / 8 : 1][2];   // the values' scales, 0 where no one sees them
            if constexpr (E8) {
#pragma unroll
                for (int t = 0; t < B / 8; ++t) {
                    const float2 ks2 = *reinterpret_cast<const float2*>(&scales[warp][st][0][8 * t + 2 * (lane & 3)]);
                    const float2 vs2 = *reinterpret_cast<const float2*>(&scales[warp][st][1][8 * t + 2 * (lane & 3)]);
                    x[t][0] *= sl2 * ks2.x;
                    x[t][1] *= sl2 * ks2.y;
                    vs[t][0] = vs2.x;
                    vs[t][1] = vs2.y;
                }
                if (!all) {   // most blocks are seen wholly
#pragma unroll
                    for (int t = 0; t < B / 8; ++t)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const bool seen = here[t / 2] && v.sees(b * B + 8 * t + 2 * (lane & 3) + c);
                            x[t][c] = seen ? x[t][c] : -INFINITY;
                            vs[t][c] = seen ? vs[t][c] : 0.f;
                        }
                }
            } else {
#pragma unroll
                for (int t = 0; t < B / 8; ++t)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        x[t][c] = all || (here[0] && v.sees(b * B + 8 * t + 2 * (lane & 3) + c)) ? x[t][c] * sl2 : -INFINITY;
            }
            if (A.c.weights && (lane >> 2) < g) {
                float* lg = A.logits + (((size_t)s * Hkv + h) * A.nbmax + i) * (size_t)(g * B) + (lane >> 2) * B + 2 * (lane & 3);
#pragma unroll
                for (int t = 0; t < B / 8; ++t) *reinterpret_cast<float2*>(lg + 8 * t) = make_float2(x[t][0], x[t][1]);
            }
            if (row >= 0) {
                if (!all) {
                    // Values that no one sees may be anything: zeros meet the weights of zero.
                    for (int r = 0; r < B; ++r)
                        if (!(here[r / kPdHalf] && v.sees(b * B + r)) && lane < (E8 ? 8 : 16))
                            ptx::st_shared_v4(src + (2 + (E8 ? 0 : lane >> 3)) * kPdTile + r * 128 + ((lane & 7) << 4), 0u, 0u, 0u, 0u);
                    ptx::fence_proxy_async_smem();   // before the stage's next TMA load
                    __syncwarp();
                }
                float t = fmaxf(x[0][0], x[0][1]);
#pragma unroll
                for (int k = 1; k < B / 8; ++k) t = fmaxf(t, fmaxf(x[k][0], x[k][1]));
                t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
                t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
                const float mn = fmaxf(m, t);
                // The sums so far refer to the new maximum; c0, c1: what E8's columns are multiplied by.
                auto rescale = [&](float c0, float c1) {
#pragma unroll
                    for (int d = 0; d < kAcc; ++d)
#pragma unroll
                        for (int c = 0; c < 4; ++c) acc[d][c] *= c & 1 ? c1 : c0;
                };
                uint32_t hi[B / 8], lo[B / 8];
                // Two slots' factors, rounded, and what that left.
                auto split = [&](int t2, float p0, float p1) {
                    hi[t2] = Half16<Operand>::pack(p0, p1);
                    const float2 r = Half16<Operand>::unpack(hi[t2]);
                    lo[t2] = Half16<Operand>::pack(p0 - r.x, p1 - r.y);
                    return r;
                };
                if constexpr (E8) {
                    const float corr = ptx::ex2(m - mn);   // 0 from kNoLogit on
                    l *= corr;
                    // Weights times scales, in x, and the largest of the head's (magnitudes compare as integers, infinities
                    // and NaN as the largest).
                    uint32_t top = 0u;
#pragma unroll
                    for (int k = 0; k < B / 8; ++k) {
                        const float p0 = ptx::ex2(x[k][0] - mn), p1 = ptx::ex2(x[k][1] - mn);
                        l += p0 + p1;
                        x[k][0] = p0 * vs[k][0];
                        x[k][1] = p1 * vs[k][1];
                        top = max(top, max(__float_as_uint(fabsf(x[k][0])), __float_as_uint(fabsf(x[k][1]))));
                    }
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    const bool unbounded = __any_sync(0xffffffffu, top >= 0x7f800000u);
                    if (unbounded) {   // the largest finite one
                        top = 0u;
#pragma unroll
                        for (int k = 0; k < B / 4; ++k) {
                            const uint32_t a = __float_as_uint(fabsf(x[k >> 1][k & 1]));
                            top = a < 0x7f800000u ? max(top, a) : top;
                        }
                        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    }
                    peak = fmaxf(peak * corr, __uint_as_float(top));
                    const float to = to_range<14>(peak);
                    if (__any_sync(0xffffffffu, mn != m || to != up)) {
                        const float f = corr * power_ratio(to, up);
                        m = mn;
                        up = to;
                        rescale(__shfl_sync(0xffffffffu, f, (lane & 3) * 8), __shfl_sync(0xffffffffu, f, (lane & 3) * 8 + 4));
                    }
#pragma unroll
                    for (int k = 0; k < B / 8; ++k) {
                        const float2 r = split(k, x[k][0] * up, x[k][1] * up);
                        if (unbounded)   // an infinite weight leaves no rest, where infinity less infinity gave NaN
                            lo[k] &= (fabsf(r.x) < INFINITY ? 0xffffu : 0u) | (fabsf(r.y) < INFINITY ? 0xffff0000u : 0u);
                    }
                } else {
                    if (__any_sync(0xffffffffu, mn != m)) {
                        const float corr = ptx::ex2(m - mn);
                        l *= corr;
                        m = mn;
                        rescale(corr, corr);
                    }
#pragma unroll
                    for (int k = 0; k < B / 8; ++k) {
                        const float p0 = ptx::ex2(x[k][0] - m), p1 = ptx::ex2(x[k][1] - m);
                        l += p0 + p1;
                        split(k, p0, p1);
                    }
                }
                // Values: row (lane & 7) + 8 (lane / 8 % 2), columns 16 dd + 8 (lane / 16).
                const int vr = (lane & 7) + (((lane >> 3) & 1) << 3);
                if constexpr (E8) {
                    // A word holds two slots' columns 2 n and 2 n + 1, n = lane / 4: rows n and n + 8 of a chunk's tile.
#pragma unroll
                    for (int dd = 0; dd < 4; ++dd)
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            uint32_t vb[4];
                            const int chunk = 2 * dd + (lane >> 4);
                            ldmatrix_x4_trans(src + (2 + half) * kPdTile + vr * 128 + ((chunk ^ (vr & 7)) << 4), vb);
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                uint32_t a[4];
#pragma unroll
                                for (int e = 0; e < 4; ++e) a[e] = e4m3_to_half2(__byte_perm(vb[2 * c + (e >> 1)], 0u, e & 1 ? 0x4431 : 0x4420));
                                Half16<Operand>::mma(acc[2 * dd + c], a[0], a[1], a[2], a[3], hi[2 * half], hi[2 * half + 1]);
                                Half16<Operand>::mma(acc[2 * dd + c], a[0], a[1], a[2], a[3], lo[2 * half], lo[2 * half + 1]);
                            }
                        }
                } else {
#pragma unroll
                    for (int dd = 0; dd < 8; ++dd) {
                        uint32_t vb[4];
                        const int chunk = (2 * dd + (lane >> 4)) & 7;
                        ldmatrix_x4_trans(src + (2 + (dd >> 2)) * kPdTile + vr * 128 + ((chunk ^ (vr & 7)) << 4), vb);
                        Half16<Operand>::mma(acc[2 * dd], hi[0], lo[0], hi[1], lo[1], vb[0], vb[1]);
                        Half16<Operand>::mma(acc[2 * dd + 1], hi[0], lo[0], hi[1], lo[1], vb[2], vb[3]);
                    }
                }
            }
            __syncwarp();   // every lane is done with the stage's tiles and row
            st = st + 1 == kPdStages ? 0 : st + 1;
            if constexpr (!kEarly) load_next();    // into the stage that the step before freed; this step's is free now
        }
        // The warp's (maximum, sum, outputs), in its free stage: the one before st.
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        float* mine = reinterpret_cast<float*>(ring + (st == 0 ? kPdStages - 1 : st - 1) * kPdStage);
        {
            const int j = lane >> 2;
            if ((lane & 3) == 0) {
                wm[warp][j] = m;
                wl[warp][j] = l;
            }
            if (lane == 0) wacc[warp] = mine;
            if constexpr (E8) {
                const float down = inverse_power(up);
                const float d0 = __shfl_sync(0xffffffffu, down, (lane & 3) * 8), d1 = __shfl_sync(0xffffffffu, down, (lane & 3) * 8 + 4);
#pragma unroll
                for (int d = 0; d < kAcc; ++d) {
                    float* const to = mine + (lane & 3) * 2 * kHeadDim + d * 16 + 2 * j;   // j = lane / 4
                    *reinterpret_cast<float2*>(to) = make_float2(acc[d][0] * d0, acc[d][2] * d0);
                    *reinterpret_cast<float2*>(to + kHeadDim) = make_float2(acc[d][1] * d1, acc[d][3] * d1);
                }
            } else {
#pragma unroll
                for (int d = 0; d < 16; ++d)
                    *reinterpret_cast<float2*>(mine + j * kHeadDim + d * 8 + 2 * (lane & 3)) =
                        make_float2(with_rest(acc[d][0], acc[d][2]), with_rest(acc[d][1], acc[d][3]));
            }
        }
        __syncthreads();
        for (int e = tid; e < g * kHeadDim; e += kPdThreads) {
            const int j = e / kHeadDim, c = e % kHeadDim;
            float M = kNoLogit;
#pragma unroll
            for (int w = 0; w < kPdWarps; ++w) M = fmaxf(M, wm[w][j]);
            float L = 0.f, O = 0.f;
#pragma unroll
            for (int w = 0; w < kPdWarps; ++w) {
                const float f = ptx::ex2(wm[w][j] - M);
                L = fmaf(f, wl[w][j], L);
                O = fmaf(f, wacc[w][e], O);
            }
            if (CL && splits > 1) {
                co[CL ? j : 0][c] = O;
                if (c == 0) {
                    cm[j] = M;
                    cl[j] = L;
                }
            } else if (CL || whole) {
                const size_t at = (size_t)s * Hq + (size_t)h * g + j;
                if constexpr (OPEN) {
                    A.own_o[at * kHeadDim + c] = O;
                    if (c == 0) A.own_ml[at] = make_float2(M, L);
                } else {
                    const float o = L > 0.f || L != L ? O / L : 0.f;
                    reinterpret_cast<T*>(A.io.out)[at * kHeadDim + c] = T(o);
                    if (c == 0) {
                        fm[j] = M;
                        finv[j] = L > 0.f || L != L ? 1.f / L : 0.f;
                    }
                }
            } else {
                const size_t slot = (size_t)blockIdx.x * 2 + (first_segment ? 0 : 1);
                A.part_o[(slot * kPdHeads + j) * kHeadDim + c] = O;
                if (c == 0) A.part_ml[slot * kPdHeads + j] = make_float2(M, L);
            }
        }
        ptx::fence_proxy_async_smem();   // the outputs lay where the next load goes
        __syncthreads();
        if constexpr (CL) {
            // A CTA of a cluster has 512 slots at most, four a thread, read while the cluster meets.
            SlotWeights<B> sw;
            sw.row = -1;
            if (!OPEN && A.c.weights && tid < len * (B / 4)) sw.load(A, s, h, v, i_begin, tid);
            if (splits > 1) {
                cg::cluster_group cluster = cg::this_cluster();
                cluster.sync();
                // Every CTA has the final sums (for its weights); it writes query heads rank, rank + splits, ...
                if (tid < g) {
                    float mc[kPdMaxCluster], M = kNoLogit, L = 0.f;
#pragma unroll
                    for (int r = 0; r < kPdMaxCluster; ++r) {
                        mc[r] = r < splits ? *cluster.map_shared_rank(&cm[tid], r) : kNoLogit;
                        M = fmaxf(M, mc[r]);
                    }
#pragma unroll
                    for (int r = 0; r < kPdMaxCluster; ++r)
                        if (r < splits) L = fmaf(ptx::ex2(mc[r] - M), *cluster.map_shared_rank(&cl[tid], r), L);
                    if (OPEN && rank == 0) A.own_ml[(size_t)s * Hq + (size_t)h * g + tid] = make_float2(M, L);
                    fm[tid] = M;
                    finv[tid] = L > 0.f || L != L ? 1.f / L : 0.f;
                }
                __syncthreads();
                for (int e = tid; rank + (e / kHeadDim) * splits < g; e += kPdThreads) {
                    const int j = rank + (e / kHeadDim) * splits, c = e % kHeadDim;
                    float O = 0.f;
#pragma unroll
                    for (int r = 0; r < kPdMaxCluster; ++r) {
                        if (r >= splits) break;
                        O = fmaf(ptx::ex2(*cluster.map_shared_rank(&cm[j], r) - fm[j]),
                                 *cluster.map_shared_rank(&co[CL ? j : 0][c], r), O);
                    }
                    const size_t at = (size_t)s * Hq + (size_t)h * g + j;
                    if constexpr (OPEN) A.own_o[at * kHeadDim + c] = O;
                    else reinterpret_cast<T*>(A.io.out)[at * kHeadDim + c] = T(O * finv[j]);
                }
                if (!OPEN && A.c.weights) sw.store(A, fm, finv);
                cluster.sync();   // no CTA leaves while another still reads its shared memory
            } else if (!OPEN && A.c.weights) {
                sw.store(A, fm, finv);
            }
            break;
        }
        if (!OPEN && A.c.weights && whole) {
            add_weights<kPdThreads, B>(A, s, h, v, i_begin, i_begin + len, fm, finv);
            __syncthreads();      // before the next segment's fm and finv
        }
        done += len;
        cur.advance(A, len);
        first_segment = false;
    }
    // Copies in flight land before the CTA may exit (a stage without one runs into the limit).
    if (failed)
        for (int i = 0; i < kPdStages; ++i) ptx::mbar_wait(&full[warp][i], (phases >> i) & 1u, 20000000ull);
}

// The pairs whose blocks several CTAs share.  Block x = 0 of (x, h, s) joins the outputs, a warp a query head, the
// others add the weights, kJoinRows slots each.  (A lane finds a share's place and sums, and eight shares' outputs are
// read at once: one thread in a loop over the 38 shares of 131072 slots took 58 us.  Six blocks resident on an
// SM: eight spill, 64 rows take the same but a window of 4096 in 16 caches 55.5 us instead of 53.6.)
template <class T, int B>
__global__ void __launch_bounds__(kJoinThreads, 6) paged_join_kernel(const __grid_constant__ PdArgs A) {
    extern __shared__ float2 share[];                 // [shares][kPdHeads] (place as an int, maximum)
    __shared__ float fm[kPdHeads], finv[kPdHeads];
    const int h = blockIdx.y, s = blockIdx.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = A.g;
    Visible<B> v;
    v.init(A, s);
    const bool weights = blockIdx.x > 0;
    const int i0 = ((int)blockIdx.x - 1) * (kJoinRows / B);
    // The lengths were complete before the kernel that this one waits for began.
    List<B> list;
    list.init(A);
    // Nothing to join: nothing is seen, finished by its CTA, or a block of slots that the sequence does not have.
    bool done = v.nb == 0 || list.whole_pairs(A) || i0 >= v.nb;
    const long long total = list.total;
    long long p0 = 0;
    int c0 = 0, c1 = 0;
    if (!done) {
        p0 = list.places_before(A, s) + (long long)h * List<B>::places(v);
        c0 = (int)quotient((p0 + kPairCost + 1) * A.ctas - 1, total);
        c1 = (int)quotient((p0 + kPairCost + v.nb) * A.ctas - 1, total);
        done = c0 == c1;
    }
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    T* const out = reinterpret_cast<T*>(A.io.out) + ((size_t)s * A.io.Hq + (size_t)h * g) * kHeadDim + lane * 4;
    if (v.nb == 0 && !weights)
        for (int j = warp; j < g; j += kJoinThreads / 32) *reinterpret_cast<uint2*>(out + j * kHeadDim) = make_uint2(0u, 0u);
    if (done) return;
    for (int j = warp; j < g; j += kJoinThreads / 32) {   // a lane a share
        float M = kNoLogit, L = 0.f;
        for (int c = lane; c <= c1 - c0; c += 32) {
            // A CTA's first segment, unless the pair begins inside its share, as it may in c0's; none if the CTA has
            // no blocks (there are fewer than CTAs).
            const int cta = c0 + c;
            int at = cta * 2;
            if (c == 0) at += share_start(total, c0, A.ctas) < p0 ? 1 : 0;
            else if (total < A.ctas && share_start(total, cta, A.ctas) == share_start(total, cta + 1, A.ctas)) at = -1;
            const float2 ml = at < 0 ? make_float2(kNoLogit, 0.f) : A.part_ml[at * kPdHeads + j];
            share[c * kPdHeads + j] = make_float2(__int_as_float(at), ml.x);
            const float m = fmaxf(M, ml.x);
            L = fmaf(L, ptx::ex2(M - m), ml.y * ptx::ex2(ml.x - m));
            M = m;
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            const float M2 = __shfl_xor_sync(0xffffffffu, M, o), L2 = __shfl_xor_sync(0xffffffffu, L, o);
            const float m = fmaxf(M, M2);
            L = fmaf(L, ptx::ex2(M - m), L2 * ptx::ex2(M2 - m));
            M = m;
        }
        // (The two halves of a pair of lanes sum in different orders: lane 0's is taken.)
        L = __shfl_sync(0xffffffffu, L, 0);
        const bool some = L > 0.f || L != L;
        if (lane == 0) {
            fm[j] = M;
            finv[j] = some ? 1.f / L : 0.f;
        }
        __syncwarp();
        if (!weights) {
            float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
            const float* part = A.part_o + (size_t)j * kHeadDim + lane * 4;
            for (int c = 0; c <= c1 - c0; c += 8) {
                float4 o[8];
                float f[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float2 sh = c + k <= c1 - c0 ? share[(c + k) * kPdHeads + j] : make_float2(__int_as_float(-1), kNoLogit);
                    const int at = __float_as_int(sh.x);
                    o[k] = at < 0 ? make_float4(0.f, 0.f, 0.f, 0.f)
                                  : *reinterpret_cast<const float4*>(part + (size_t)at * (kPdHeads * kHeadDim));
                    f[k] = ptx::ex2(sh.y - M);
                }
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    O = make_float4(fmaf(f[k], o[k].x, O.x), fmaf(f[k], o[k].y, O.y), fmaf(f[k], o[k].z, O.z), fmaf(f[k], o[k].w, O.w));
            }
            *reinterpret_cast<uint2*>(out + j * kHeadDim) = some ? make_uint2(Half16<T>::pack(O.x / L, O.y / L), Half16<T>::pack(O.z / L, O.w / L))
                                                  : make_uint2(0u, 0u);
        }
    }
    if (!weights) return;
    __syncthreads();
    add_weights<kJoinThreads, B>(A, s, h, v, i0, min(v.nb, i0 + kJoinRows / B), fm, finv);
}

// shared_decode: what the shares of a group's prefix and those of the sequence's own slots sum up to.  Block x = 0 of
// (x, h, s) writes the outputs, a warp a query head, the others add the weights, kJoinRows slots each.  Sums lie as rows of
// 128 values behind one another: the CTAs' shares of pairs, whole pairs, the prefixes' shares.  A lane reads a share's
// maximum and sum, and eight shares' rows are read at once.
// NT: threads, a warp for each of four heads, or of eight (64 rows of 7 heads behind 4096 slots 34.4 us with eight warps, 35.1 with
// four; 160 of 4 heads 163 and 157).
// one_each: every pair's own sums are whole (a cluster each); else as the list of blocks says.
template <class T, int NT, int B>
__global__ void __launch_bounds__(NT, 768 / NT) shared_join_kernel(const __grid_constant__ PdArgs A, int prefix_ctas, bool one_each) {
    __shared__ float fm[kPdHeads], finv[kPdHeads];
    const int h = blockIdx.y, s = blockIdx.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = A.g;
    // The lengths were complete before the call.
    Visible<B> v;
    v.init(A, s);
    const bool weights = blockIdx.x > 0;
    const int i0 = ((int)blockIdx.x - 1) * (kJoinRows / B);
    const int own_rows = A.ctas * 2 * kPdHeads, prefix_rows = own_rows + A.io.batch * A.io.Hq;
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    if (weights && i0 >= v.nb) return;
    int own = v.nb ? 1 : 0, c0 = 0;   // the pair's own shares, of CTAs c0 on
    long long total = 0, p0 = 0;
    bool whole = true;
    if (!one_each && v.nb) {
        const longlong2 all = A.own_plan[A.io.batch];
        total = all.x;
        whole = all.y != 0;
        p0 = A.own_plan[s].x + (long long)h * List<B>::places(v);
        if (!whole) {
            c0 = (int)quotient((p0 + kPairCost + 1) * A.ctas - 1, total);
            own = (int)quotient((p0 + kPairCost + v.nb) * A.ctas - 1, total) - c0 + 1;
            whole = own == 1;
        }
    }
    const PrefixParts parts(A.prefix_plan[s], h, prefix_ctas);
    const int n = own + parts.n;
    for (int j = warp; j < g; j += NT / 32) {
        float M = kNoLogit, L = 0.f;
        float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k0 = 0; k0 < n; k0 += 32) {
            const int k = k0 + lane;
            int row = -1;
            if (k < own) {
                const int cta = c0 + k;
                if (whole) row = own_rows + s * A.io.Hq + h * g + j;
                else if (k == 0) row = (cta * 2 + (share_start(total, c0, A.ctas) < p0 ? 1 : 0)) * kPdHeads + j;
                else if (total >= A.ctas || share_start(total, cta, A.ctas) < share_start(total, cta + 1, A.ctas)) row = cta * 2 * kPdHeads + j;
            } else if (k < n) {
                row = parts.row(k - own);
                if (row >= 0) row += prefix_rows + j;
            }
            const float2 ml = row < 0 ? make_float2(kNoLogit, 0.f) : A.part_ml[row];
            float m = ml.x;
#pragma unroll
            for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            m = fmaxf(m, M);
            const float f = ptx::ex2(M - m), w = row < 0 ? 0.f : ptx::ex2(ml.x - m);
            float l = w * ml.y;
#pragma unroll
            for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
            L = fmaf(L, f, l);
            M = m;
            if (weights) continue;
            O = make_float4(O.x * f, O.y * f, O.z * f, O.w * f);
            for (int e0 = 0; e0 < min(32, n - k0); e0 += 8) {
                float4 o[8];
                float wk[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int from = __shfl_sync(0xffffffffu, row, e0 + e);
                    wk[e] = __shfl_sync(0xffffffffu, w, e0 + e);
                    o[e] = from < 0 ? make_float4(0.f, 0.f, 0.f, 0.f)
                                    : reinterpret_cast<const float4*>(A.part_o + (size_t)from * kHeadDim)[lane];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    O = make_float4(fmaf(wk[e], o[e].x, O.x), fmaf(wk[e], o[e].y, O.y), fmaf(wk[e], o[e].z, O.z), fmaf(wk[e], o[e].w, O.w));
            }
        }
        // (The lanes sum in different orders: lane 0's sum is taken.)
        L = __shfl_sync(0xffffffffu, L, 0);
        const bool some = L > 0.f || L != L;
        if (lane == 0) {
            fm[j] = M;
            finv[j] = some ? 1.f / L : 0.f;
        }
        if (!weights)
            reinterpret_cast<uint2*>(reinterpret_cast<T*>(A.io.out) + ((size_t)s * A.io.Hq + (size_t)h * g + j) * kHeadDim)[lane] =
                some ? make_uint2(Half16<T>::pack(O.x / L, O.y / L), Half16<T>::pack(O.z / L, O.w / L)) : make_uint2(0u, 0u);
    }
    if (!weights) return;
    __syncthreads();
    add_weights<NT, B>(A, s, h, v, i0, min(v.nb, i0 + kJoinRows / B), fm, finv);
}

size_t round16(size_t x) { return (x + 15) & ~size_t(15); }

int share_ctas(int num_sms) { return kPdCtasPerSm * num_sms; }

// one_each: set to whether each pair is finished by a cluster.
template <class T, bool E8, bool OPEN>
cudaError_t launch_pairs(const PdArgs& a, cudaStream_t st, bool* one_each) {
    constexpr int B = kPdBlock<E8>;
    // CTAs of a pair: the largest cluster that fits the device's resident CTAs in one wave, with
    // two blocks a warp and more; taken where that leaves a CTA 32 blocks and less (a quarter of
    // one a thread for the weights), else the list of all blocks.  Measured with weights, 8 KV
    // heads, in us by cluster and by list: one row of 4096 slots 13.3, of 8192 (list) 16.3; 512
    // rows of 100 to 300 slots (a CTA each) 110 and 147; 40 of 1000 slots (two CTAs each, more than a
    // wave) 47.7 and 39.5, 256 of 1500 365 and 272.
    const int pairs = a.io.batch * a.io.Hkv;
    int splits = 1;
    while (splits < kPdMaxCluster && (long long)pairs * splits * 2 <= a.ctas && a.nbmax >= kPdWarps * 2 * splits) splits *= 2;
    *one_each = a.nbmax * (B / 4) <= kPdThreads * splits;
    if (*one_each) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(splits, a.io.Hkv, a.io.batch);
        cfg.blockDim = dim3(kPdThreads);
        cfg.dynamicSmemBytes = kPdSmem;
        cfg.stream = st;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = splits;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        return cudaLaunchKernelEx(&cfg, paged_decode_kernel<T, true, E8, OPEN>, a);
    }
    return launch_prio(paged_decode_kernel<T, false, E8, OPEN>, dim3(a.ctas), dim3(kPdThreads), kPdSmem, st, 0, true, a);
}

// Blocks of a join that add the weights of a pair.
int weight_blocks(const PdArgs& a, int B) { return a.c.weights ? (a.nbmax * B + kJoinRows - 1) / kJoinRows : 0; }

template <class T, bool E8>
cudaError_t launch_typed(const PdArgs& a, cudaStream_t st) {
    constexpr int B = kPdBlock<E8>;
    bool one_each = false;
    const cudaError_t e = launch_pairs<T, E8, false>(a, st, &one_each);
    if (e != cudaSuccess || one_each) return e;
    return launch_prio(paged_join_kernel<T, B>, dim3(1 + weight_blocks(a, B), a.io.Hkv, a.io.batch), dim3(kJoinThreads),
                       a.ctas * kPdHeads * sizeof(float2), st, 0, true, a);
}

template <class T, bool E8>
cudaError_t launch_shared_typed(const PdArgs& a, const PrefixIO& px, int num_sms, cudaStream_t st) {
    constexpr int B = kPdBlock<E8>;
    bool one_each = false;
    cudaError_t e = launch_pairs<T, E8, true>(a, st, &one_each);
    if (e == cudaSuccess) e = launch_prefix(px, num_sms, st);
    if (e != cudaSuccess) return e;
    auto join = [&](auto kernel, int threads) {
        return launch_prio(kernel, dim3(1 + weight_blocks(a, B), a.io.Hkv, a.io.batch), dim3(threads), 0, st, 0, true, a,
                           num_sms, one_each);
    };
    return a.g <= 4 ? join(shared_join_kernel<T, 128, B>, 128) : join(shared_join_kernel<T, 256, B>, 256);
}

// Most blocks of B slots that a sequence of up to max_len slots has in sight.
int visible_blocks(int B, int max_len, int window, int sinks) {
    const int all = (max_len + B - 1) / B;
    if (!window) return all;
    // A window ends and begins inside a block.
    const long long some = (long long)window / B + 2 + (std::min(sinks, max_len) + B - 1) / B;
    return (int)std::min<long long>(all, some);
}

}  // namespace

size_t paged_decode_scratch(int batch, int Hq, int max_len, int window, int sinks, bool weights, bool e8, int num_sms) {
    const int B = e8 ? kPdBlock<true> : kPdBlock<false>;
    const size_t slots = (size_t)share_ctas(num_sms) * 2 * kPdHeads;
    size_t b = round16(slots * kHeadDim * sizeof(float)) + round16(slots * sizeof(float2));
    if (weights) b += (size_t)batch * Hq * visible_blocks(B, max_len, window, sinks) * B * sizeof(float);
    return b;
}

// Rows of sums: the CTAs' shares, whole pairs, and the prefixes'.
size_t shared_decode_scratch(int batch, int Hq, int max_len, bool weights, bool e8, int num_sms) {
    const int B = e8 ? kPdBlock<true> : kPdBlock<false>;
    const size_t rows = (size_t)share_ctas(num_sms) * 2 * kPdHeads + (size_t)batch * Hq * 2 + (size_t)2 * kPrefixTile * num_sms;
    size_t b = rows * kHeadDim * sizeof(float) + round16(rows * sizeof(float2)) + batch * sizeof(PrefixPlan) + (batch + 1) * sizeof(longlong2);
    if (weights) b += (size_t)batch * Hq * visible_blocks(B, max_len, 0, 0) * B * sizeof(float);
    return b;
}

cudaError_t configure_paged_decode() {
    cudaError_t e = cudaSuccess;
    auto one = [&](auto kernel) {
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPdSmem);
    };
    auto both = [&](auto type) {
        using T = decltype(type);
        one(paged_decode_kernel<T, true, false, false>);
        one(paged_decode_kernel<T, false, false, false>);
        one(paged_decode_kernel<T, true, true, false>);
        one(paged_decode_kernel<T, false, true, false>);
        one(paged_decode_kernel<T, true, false, true>);
        one(paged_decode_kernel<T, false, false, true>);
        one(paged_decode_kernel<T, true, true, true>);
        one(paged_decode_kernel<T, false, true, true>);
    };
    both(__nv_bfloat16{});
    both(__half{});
    return e;
}

namespace {

// Everything but the places in scratch.
cudaError_t fill_args(PdArgs& a, const PagedDecodeIO& io, const PagedCacheView& c, int num_sms) {
    // Rows of 8 bits as 64 elements of 16: the copies only move them.
    const bool e8 = c.k_scales != nullptr;
    const uint64_t dims[2] = {(uint64_t)(e8 ? kHeadDim / 2 : kHeadDim), ((uint64_t)c.num_pages * io.Hkv) << c.log_page};
    const uint64_t strides[1] = {dims[0] * 2};
    a.box = e8 && c.log_page >= 5 ? kPdBlock<true> : kPdHalf;
    const uint32_t box[2] = {64, (uint32_t)a.box};
    cudaError_t e = encode_tensor_map(&a.kmap, c.dtype, 2, c.k, dims, strides, box);
    if (e == cudaSuccess) e = encode_tensor_map(&a.vmap, c.dtype, 2, c.v, dims, strides, box);
    a.c = c;
    a.io = io;
    a.g = io.Hq / io.Hkv;
    a.sl2 = io.scale * 1.4426950408889634f;
    a.fault = test_fault() == 4 ? 1 : 0;
    a.ctas = share_ctas(num_sms);
    const long long pairs = (long long)io.batch * io.Hkv;
    a.pairs = pairs <= a.ctas && pairs * 4 >= a.ctas * 3ll ? (int)pairs : 0;
    a.nbmax = visible_blocks(e8 ? kPdBlock<true> : kPdBlock<false>, io.max_len, io.window, io.sinks);
    return e;
}

}  // namespace

cudaError_t launch_paged_decode(const PagedDecodeIO& io, const PagedCacheView& c, int num_sms, cudaStream_t st) {
    PdArgs a{};
    const cudaError_t e = fill_args(a, io, c, num_sms);
    if (e != cudaSuccess) return e;
    const size_t slots = (size_t)a.ctas * 2 * kPdHeads;
    char* p = static_cast<char*>(io.scratch);
    a.part_o = reinterpret_cast<float*>(p);
    p += round16(slots * kHeadDim * sizeof(float));
    a.part_ml = reinterpret_cast<float2*>(p);
    p += round16(slots * sizeof(float2));
    a.logits = reinterpret_cast<float*>(p);
    auto launch = [&](auto type) {
        using T = decltype(type);
        return c.k_scales ? launch_typed<T, true>(a, st) : launch_typed<T, false>(a, st);
    };
    return c.dtype == 1 ? launch(__half{}) : launch(__nv_bfloat16{});
}

cudaError_t launch_shared_decode(const PagedDecodeIO& io, const PagedCacheView& c, const PrefixIO& prefix, int num_sms, cudaStream_t st) {
    PdArgs a{};
    const cudaError_t e = fill_args(a, io, c, num_sms);
    if (e != cudaSuccess) return e;
    const size_t shares = (size_t)a.ctas * 2 * kPdHeads, pairs = (size_t)io.batch * io.Hq;
    const size_t rows = shares + 2 * pairs + (size_t)2 * kPrefixTile * num_sms;
    a.part_o = static_cast<float*>(io.scratch);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + rows * kHeadDim);
    a.own_o = a.part_o + shares * kHeadDim;
    a.own_ml = a.part_ml + shares;
    PrefixIO px = prefix;
    px.plan = reinterpret_cast<PrefixPlan*>(reinterpret_cast<char*>(a.part_ml) + round16(rows * sizeof(float2)));
    a.prefix_plan = px.plan;
    a.own_plan = reinterpret_cast<longlong2*>(px.plan + io.batch);
    a.logits = reinterpret_cast<float*>(a.own_plan + io.batch + 1);
    px.part_o = a.own_o + pairs * kHeadDim;
    px.part_ml = a.own_ml + pairs;
    auto launch = [&](auto type) {
        using T = decltype(type);
        return c.k_scales ? launch_shared_typed<T, true>(a, px, num_sms, st) : launch_shared_typed<T, false>(a, px, num_sms, st);
    };
    return c.dtype == 1 ? launch(__half{}) : launch(__nv_bfloat16{});
}

}  // namespace kvec
