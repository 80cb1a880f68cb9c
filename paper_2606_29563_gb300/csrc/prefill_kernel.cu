// Causal attention of packed sequences with an optional sliding window and first tokens
// that stay visible, and each row's log-sum-exp:
//   s = scale log2(e) Q K^T,  out = sum_t 2^(s_t - m) v_t / l,  l = sum_t 2^(s_t - m),
//   lse = ln 2 (m + log2 l),
// over the keys t <= p that a row at position p sees (t > p - window or t < sinks).
//
// A CTA owns two tiles of 128 rows; a row is a (query, query head) pair, the g query heads
// of one KV head side by side, so that one query fills g rows and both tiles read the same
// K and V.  It walks the 128-key blocks that any of its rows sees:
//   warps 0-3, 4-7  softmax of tile 0 and 1, one thread a row: S from TMEM, running sum, the
//                   weights back to TMEM as 16-bit values over S; at the end the outputs;
//   warp 8          TMA: the query rows once, then K and V blocks through a ring; finds the items of
//                   sequences of different lengths;
//   warps 9, 10     tcgen05.mma, a warp for each tile: O += P V (P from TMEM, V column-major
//                   from shared memory), then the next S = Q K^T (both from shared memory), in
//                   turns, so that one tile's softmax runs beside the other's products;
//   warp 11         blocks that some row does not see wholly: zeroes what V holds there of
//                   infinities and NaN, which a weight of zero would not keep out.  What a row
//                   sees of them is added at the end.
// A row's weights refer to a maximum m that need not be the largest: it is that of the first
// block in which the row sees a key, and moves only when the weights of a block sum up to 2^14
// (kMostWeight), so that no block waits for a maximum and O is scaled in TMEM once in a while.
// Results do not depend on m: 2^(s - m) keeps its relative precision, and so does l.
// The weights meet V rounded to its type, as the tensor cores take both operands of one type; their
// sum l is that of the unrounded ones.  That adds half a step of the type to the output's own
// rounding (error against 64 bits 2.2e-3 of the output for 1.6e-3 in bf16, 2.6e-4 for 2.1e-4 in
// fp16); a second product with what the rounding left would take half as much tensor time again.
//
// Bound by the power limit in long runs, and by the products' chain before it: a block of both
// tiles takes 2048 cycles of the tensor pipe (32 products of 64 cycles, which is what they take
// when nothing waits) and about 2700 in all, as a tile's softmax (S read 60, exponentials 2 x
// 370, weights written and handed over 250 cycles) and its turn's waits outlast the other tile's
// 1024.  (Without any exponential 8192 tokens take 317 us instead of 333.)  Measured, 32 query
// and 8 KV heads, bf16, in CUDA graphs of a few calls: 32768 tokens 5.15 ms, 1709 TFLOP/s;
// 8192 tokens 330 us, 1667 TFLOP/s (89 % of the measured cuBLAS burst), in a run of seconds 365 us
// at 1830 MHz and 1370 W, 1506 TFLOP/s (a cuBLAS product of 8192^3 beside it 1690 at 1430 MHz); 16384
// tokens with a window of 2048 and 4 first tokens 389 us, 1327 TFLOP/s of visible pairs (18 blocks an item
// for 16 of keys seen); 8192 and 5001 tokens together 464 us, 1627 TFLOP/s.  What that took, 8192 tokens in us:
// S in registers without spills 451, items one behind the other in persistent CTAs 445, no
// maximum pass 421, waits of one poll 406, 32-byte stores 398, stages stepped 390, whole blocks
// of weights handed over at once 375, a warp that issues for each tile 349, the registers that
// this one needs no longer given to the softmax 334, the next item looked up before its turn 331,
// no branch between most turns' products 328.
// Slower: outputs by a warpgroup of their own (396 for 375: 64 registers for the others spill),
// halves of blocks left out where no row sees them (425 for 390: the branches stand between the
// products), products of 16 keys for a block of few first tokens (348 for 331, and in turns of
// their own no gain: 394 for 391 with the window).
#include <algorithm>
#include <type_traits>

#include "half_types.cuh"
#include "kvec_internal.cuh"
#include "sm100_ptx.cuh"

namespace kvec {

namespace {

constexpr int kPfTile = 128;                        // rows of a tile, keys of a block
constexpr int kPfHalf = kPfTile * 128;              // bytes of 128 rows x 64 columns
constexpr int kPfBuf = 2 * kPfHalf;                 // a tile or block: 32 KB
constexpr int kPfStages = 5;
constexpr int kPfItems = 4;                         // items handed out and not yet taken by every warp
constexpr int kPfThreads = 384;
constexpr uint32_t kPfTmem = 512;                   // S0 | S1 | O0 | O1, 128 columns each
// Registers of a thread: at launch (the most that 384 threads may have), and after the split.
// The compiler spills one or two words, and eight in the variant of ragged lengths (-Xptxas -v).
constexpr int kPfRegs = 168, kPfSoftmaxRegs = 216, kPfOtherRegs = 72;
static_assert(256 * kPfSoftmaxRegs + 128 * kPfOtherRegs <= kPfThreads * kPfRegs, "the split fits what the block was launched with");
// A row's weights of a block that sum up to less are taken as they are; fp16 holds them.
constexpr float kMostWeight = 16384.f;
// The maximum before the first visible logit, finite: 2^(-inf - it) is 0.
constexpr float kNoLogit = -3.402823466e38f;

// Division of 0 <= x < 2^30 by a d below 2^21 that the host knows: x ceil(2^52 / d) / 2^52 is
// off by less than x d / 2^52 / d < 1 / d.
struct Divisor {
    unsigned long long m;
    __host__ void set(int d) { m = ((1ull << 52) + d - 1) / d; }
    __device__ __forceinline__ int divide(int x) const { return (int)__umul64hi((unsigned long long)x << 12, m); }
};

struct PfArgs {
    CUtensorMap qmap, kmap, vmap;
    PrefillIO io;
    int g, nq;       // query heads of a KV head, queries of a tile
    int pairs;       // tile pairs of the longest sequence
    int parts;       // of a pair's blocks, each an item (1: none are split)
    int items;       // pairs * batch * Hkv * parts: places for items, of which a short sequence leaves some unused
    float* part_o;   // [items][2][128][128] a part's sums P V, by row
    float2* part_ml; // [items][2][128] (m, l) of the rows
    Divisor by_per, by_heads;   // batch * Hkv, Hkv
    float sl2;
    int fault;       // test of the error path (kvec_set_test_fault): no S is ever complete
};

// What a CTA works on: tiles 2 p and 2 p + 1 of sequence s, KV head h.
struct alignas(16) Item {
    int h, q0, k0;                // first rows of the sequence
    int a, b;                     // the pair's queries [a, b) of the sequence
    int tiles;                    // 1 or 2
    int off;                      // position of query 0
    int nsink, lo;                // the blocks seen: 0 .. nsink - 1, then from lo on
    int i0, n;                    // of them this item's part: the n from the i0-th on (-1: the work is done)
    int place;                    // among A.items
    int whole_lo, whole_hi;       // the blocks from the whole_lo-th to before the whole_hi-th are seen by every row
    __device__ __forceinline__ int block(int i) const { return i0 + i < nsink ? i0 + i : lo + i0 + i - nsink; }
    __device__ __forceinline__ bool edge(int i) const { return i < whole_lo || i >= whole_hi; }
};

struct PfBarriers {
    uint64_t full[kPfStages], empty[kPfStages];
    uint64_t clean[kPfStages];   // the cleaning warp has passed the stage
    uint64_t q_full, q_empty, mma_done;
    uint64_t s_full[2], p_full[2], o_done[2];   // o_done: of an item
    uint64_t turn[2];            // a tile's products may be issued
    uint64_t item_full[kPfItems], item_empty[kPfItems];
    Item items[kPfItems];        // handed from the TMA warp to the others
    uint32_t tmem_base;
    volatile int abort_flag;
    volatile int unbounded;      // a block of partial sight held an infinity or NaN in V (of any item so far)
};

constexpr int kPfSmem = 1024 + (2 + kPfStages) * kPfBuf + (int)sizeof(PfBarriers);

// Where a sequence's queries and keys begin, and how many there are.
struct Rows {
    int q0, Lq, k0, Lk;
    __device__ __forceinline__ Rows(const PfArgs& A, int s) : q0(0), Lq(0), k0(0), Lk(0) {
        if (s >= A.io.batch) return;
        auto clamped = [](int v, int most) { return min(max(v, 0), most); };
        q0 = clamped(__ldg(&A.io.cu_q[s]), A.io.total_q);
        k0 = clamped(__ldg(&A.io.cu_k[s]), A.io.total_k);
        Lq = max(clamped(__ldg(&A.io.cu_q[s + 1]), A.io.total_q) - q0, 0);
        Lk = max(clamped(__ldg(&A.io.cu_k[s + 1]), A.io.total_k) - k0, 0);
    }
};

// Part `part` of what KV head h of pair p of sequence s sees; false: the sequence has no such pair.
template <bool PARTS>
__device__ __forceinline__ bool make_item(const PfArgs& A, int p, int s, const Rows& r, int h, int part, Item& w) {
    const PrefillIO& io = A.io;
    w.h = h;
    w.place = (((A.pairs - 1 - p) * io.batch + s) * io.Hkv + h) * A.parts + part;
    w.q0 = r.q0;
    w.k0 = r.k0;
    w.a = 2 * p * A.nq;
    if (w.a >= r.Lq) return false;
    w.b = min(w.a + 2 * A.nq, r.Lq);
    w.tiles = w.b - w.a > A.nq ? 2 : 1;
    w.off = r.Lk - r.Lq;
    const int pa = w.off + w.a, pb = w.off + w.b - 1;    // first and last position
    w.nsink = w.lo = w.i0 = w.n = 0;
    if (pb >= 0) {
        w.lo = io.window ? max(pa - io.window + 1, 0) / kPfTile : 0;
        w.nsink = min((min(io.sinks, r.Lk) + kPfTile - 1) / kPfTile, w.lo);
        w.n = w.nsink + pb / kPfTile + 1 - w.lo;
        if constexpr (PARTS) {
            const int all = w.n;
            w.i0 = all * part / A.parts;
            w.n = all * (part + 1) / A.parts - w.i0;
        }
    }
    // Keys [pb - window + 1, pa] are seen by every row.
    const int first = io.window ? max(pb - io.window + 1, 0) : 0;
    w.whole_lo = max((first + kPfTile - 1) / kPfTile, w.lo) - w.lo + w.nsink - w.i0;
    w.whole_hi = ((pa + 1) >> 7) - w.lo + w.nsink - w.i0;
    static_assert(kPfTile == 128, "the shift");
    return true;
}

// The item of a place; false: there is none.
template <bool PARTS>
__device__ __forceinline__ bool item_at(const PfArgs& A, int x, Item& w) {
    if (x >= A.items) return false;
    int part = 0;
    if constexpr (PARTS) {
        part = x % A.parts;
        x /= A.parts;
    }
    const int per = A.io.batch * A.io.Hkv;
    const int top = A.by_per.divide(x);
    x -= top * per;
    const int s = A.by_heads.divide(x);
    return make_item<PARTS>(A, A.pairs - 1 - top, s, Rows(A, s), x - s * A.io.Hkv, part, w);
}

// Of every gridDim.x items (or places for them) a CTA takes one, in turns from the front and
// from the back: they cost less and less, so that the shares are even.
__device__ __forceinline__ int item_of(int turn) {
    const int c = blockIdx.x, G = gridDim.x;
    return turn * G + (turn & 1 ? G - 1 - c : c);
}

// ptx::warp_wait; a phase that is over, the usual case, costs one poll and one vote.
__device__ __forceinline__ bool pf_wait(uint64_t* bar, uint32_t parity, const volatile int* abort) {
    return __all_sync(0xffffffffu, ptx::mbar_try_wait(bar, parity)) || ptx::warp_wait(bar, parity, abort);
}

// The n lowest bits, n clamped to [0, 32].
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

// The items in order: the last pairs, which see the most keys, first, then by sequence and head,
// without the pairs that shorter sequences lack.  One warp walks them: pairs lo <= p < hi are
// there in the same `count` sequences, those with hi pairs and more, and make up a run of items
// from the base-th on.  A lane keeps one of the first 32 sequences.
struct Finder {
    const PfArgs& A;
    const int lane;
    const Rows mine;
    int hi, lo, count = 0, base = 0;
    __device__ __forceinline__ Finder(const PfArgs& args, int l)
        : A(args), lane(l), mine(args, l), hi(args.pairs), lo(args.pairs) {}
    __device__ __forceinline__ int pairs_of(int s) const {
        const int Lq = s < 32 ? mine.Lq : Rows(A, s).Lq;
        return min((int)(((unsigned)Lq + 2u * A.nq - 1u) / (2u * A.nq)), A.pairs);
    }
    // The x-th item, x larger than in the calls before.
    __device__ __forceinline__ bool find(int x, Item& w) {
        const int each = A.io.Hkv;   // items of a pair
        while (x - base >= (hi - lo) * count * each) {
            if (lo == 0) return false;
            base += (hi - lo) * count * each;
            hi = lo;
            count = 0;
            int below = 0;
#pragma unroll 1
            for (int s = lane; s - lane < A.io.batch; s += 32) {
                const int p = pairs_of(s);
                count += __popc(__ballot_sync(0xffffffffu, p >= hi));
                below = max(below, p < hi ? p : 0);
            }
            lo = __reduce_max_sync(0xffffffffu, below);
        }
        int k = (x - base) / each;
        const int h = x - base - k * each;
        const int level = k / count;
        k -= level * count;   // the k-th of the sequences
#pragma unroll 1
        for (int s = lane; s - lane < A.io.batch; s += 32) {
            const uint32_t there = __ballot_sync(0xffffffffu, pairs_of(s) >= hi);
            const uint32_t it = __ballot_sync(0xffffffffu, (there >> lane & 1u) && __popc(there & low_bits(lane)) == k);
            if (it) {
                const int from = __ffs(it) - 1;
                Rows r = mine;
                if (s >= 32) r = Rows(A, s - lane + from);
                r.q0 = __shfl_sync(0xffffffffu, r.q0, from);
                r.Lq = __shfl_sync(0xffffffffu, r.Lq, from);
                r.k0 = __shfl_sync(0xffffffffu, r.k0, from);
                r.Lk = __shfl_sync(0xffffffffu, r.Lk, from);
                return make_item<false>(A, hi - 1 - level, s - lane + from, r, h, 0, w);
            }
            k -= __popc(there);
        }
        return false;   // never: `count` sequences are there
    }
};

struct NoFinder {
    __device__ __forceinline__ NoFinder(const PfArgs&, int) {}
};

// 32 bytes to a 32-byte aligned place.
__device__ __forceinline__ void st_global_v8(void* p, const uint32_t* r) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                 "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;\n" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// 32 columns of 32-bit values to this warp's TMEM lanes.
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};\n" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }

// D += A B with A (128 rows x 16) in TMEM and B in shared memory.
__device__ __forceinline__ void mma_tmem_a(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n" ::"r"(d),
        "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Shared-memory descriptor of a V block as the B operand of O += P V: columns (the values'
// dimensions) contiguous, 64 to a 128-byte swizzled row; the other 64 a half further on,
// eight keys every 1024 bytes.
__device__ __forceinline__ uint64_t smem_desc_mn_sw128(uint32_t saddr) {
    uint64_t d = 0;
    d |= (uint64_t)((saddr >> 4) & 0x3FFF);
    d |= (uint64_t)(kPfHalf >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

template <class T>
constexpr uint32_t kType = 1u;         // operand type of the instruction descriptor: bf16
template <>
constexpr uint32_t kType<__half> = 0u;

// fp32 accumulators, M = N = 128; b_mn: B's columns contiguous.
template <class T>
__device__ __forceinline__ constexpr uint32_t pf_idesc(bool b_mn) {
    return (1u << 4) | (kType<T> << 7) | (kType<T> << 10) | (b_mn ? 1u << 16 : 0u) | ((kPfTile >> 3) << 17) |
           ((kPfTile >> 4) << 24);
}

// The larger magnitude of each half (its sign is either), NaN if one is.
template <class T>
__device__ __forceinline__ uint32_t largest(uint32_t a, uint32_t b) {
    uint32_t d;
    if constexpr (!kType<T>)
        asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    else
        asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
template <class T>
__device__ __forceinline__ uint32_t unbounded_mask(uint32_t w) {   // the halves that are infinite or NaN
    constexpr uint32_t e = kType<T> ? 0x7f80u : 0x7c00u;
    return ((w & e) == e ? 0xffffu : 0u) | (((w >> 16) & e) == e ? 0xffff0000u : 0u);
}

// Persistent: no role waits for an item's end: the next one's K and V follow through the ring,
// its first S is formed behind the last products of this one, while the softmax warps write
// their outputs.
// PARTS: a pair's blocks are divided into several items, which leave sums for prefill_join_kernel.
// RAGGED: the CTAs share out the items, which the TMA warp finds and hands to the others, instead
// of the places for them, of which shorter sequences leave many unused.
template <class T, bool PARTS, bool RAGGED>
__global__ void __launch_bounds__(kPfThreads, 1) prefill_kernel(const __grid_constant__ PfArgs A) {
    static_assert(!(PARTS && RAGGED), "items that are parts have a place each");
    extern __shared__ uint8_t pf_smem_raw[];
    // 1024-byte alignment for the swizzled operand tiles.
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(pf_smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sQ = smem;
    uint8_t* ring = sQ + 2 * kPfBuf;
    PfBarriers* bars = reinterpret_cast<PfBarriers*>(ring + kPfStages * kPfBuf);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        ptx::prefetch_tensormap(&A.qmap);
        ptx::prefetch_tensormap(&A.kmap);
        ptx::prefetch_tensormap(&A.vmap);
        for (int i = 0; i < kPfStages; ++i) {
            ptx::mbar_init(&bars->full[i], 1);
            ptx::mbar_init(&bars->empty[i], 3);    // the products of both tiles, and the cleaning warp
            ptx::mbar_init(&bars->clean[i], 1);
        }
        ptx::mbar_init(&bars->q_full, 1);
        ptx::mbar_init(&bars->q_empty, 2);
        ptx::mbar_init(&bars->mma_done, 2);
        for (int t = 0; t < 2; ++t) {
            ptx::mbar_init(&bars->s_full[t], A.fault ? 2 : 1);   // 2, for a test of the waits: never complete
            ptx::mbar_init(&bars->p_full[t], 4);   // one arrival per warp of the tile
            ptx::mbar_init(&bars->o_done[t], 1);
            ptx::mbar_init(&bars->turn[t], 1);
        }
        for (int i = 0; i < kPfItems; ++i) {
            ptx::mbar_init(&bars->item_full[i], 1);
            ptx::mbar_init(&bars->item_empty[i], kPfThreads / 32 - 1);   // every warp but the one that hands out
        }
        bars->abort_flag = 0;
        bars->unbounded = 0;
        ptx::fence_barrier_init();
    }
    if (warp == 9) {
        ptx::tmem_alloc(&bars->tmem_base, kPfTmem);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    const uint32_t tmem = (uint32_t)ptx::warp_uniform((int)bars->tmem_base);
    const volatile int* const abort = &bars->abort_flag;
    const int sinks = A.io.sinks;
    bool stop = false;
    auto give_up = [&]() {
        if (stop && lane == 0) {
            bars->abort_flag = 1;
            atomicExch(A.io.err, 3);
        }
    };
    // The next item, the same for every warp; false: none is left.
    int taken = 0;
    const int turns = (A.items + gridDim.x - 1) / gridDim.x;
    auto take_item = [&](Item& w) {
        if constexpr (!RAGGED) {
            while (taken < turns)
                if (item_at<PARTS>(A, item_of(taken++), w)) return true;
            return false;
        }
        const int slot = taken % kPfItems;
        if (stop || !pf_wait(&bars->item_full[slot], (taken / kPfItems) & 1, abort)) {
            stop = true;
            return false;
        }
        w = bars->items[slot];
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&bars->item_empty[slot]);
        ++taken;
        return w.n >= 0;
    };
    // A softmax thread holds a row of S: registers move to the two softmax warpgroups.
    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kPfOtherRegs));
        int x = 0;   // loads of K and V so far: load x goes to stage x % kPfStages
        if (warp == 8) {
            // -------------------------------------------------------- TMA
            const uint64_t policy = ptx::policy_evict_normal();
            int qloads = 0;
            // The CTA's item of a turn, handed out while the one before is loaded.
            auto hand_out = [&, finder = std::conditional_t<RAGGED, Finder, NoFinder>(A, lane)](int turn) mutable {
                if constexpr (RAGGED) {
                    const int slot = turn % kPfItems;
                    Item w{};
                    if (!finder.find(item_of(turn), w)) w.n = -1;
                    if (turn >= kPfItems && !pf_wait(&bars->item_empty[slot], (turn / kPfItems - 1) & 1, abort)) stop = true;
                    if (!stop && lane == 0) {
                        bars->items[slot] = w;
                        ptx::mbar_arrive(&bars->item_full[slot]);
                    }
                    __syncwarp();
                }
            };
            hand_out(0);
            for (int turn = 0; !stop; ++turn) {
                Item w{};
                if constexpr (RAGGED) {
                    w = bars->items[turn % kPfItems];
                    if (w.n < 0) break;
                } else if (!take_item(w)) {
                    break;
                }
                if (w.n == 0) {
                    hand_out(turn + 1);
                    continue;
                }
                auto load_kv = [&](int y) {   // load y of the item: K and V blocks alternate
                    const int st = x % kPfStages, round = x / kPfStages;
                    if (round > 0 && !pf_wait(&bars->empty[st], (round - 1) & 1, abort)) {
                        stop = true;
                        return;
                    }
                    if (ptx::elect_one()) {
                        const CUtensorMap* map = y & 1 ? &A.vmap : &A.kmap;
                        uint8_t* dst = ring + st * kPfBuf;
                        const int row = w.k0 + w.block(y >> 1) * kPfTile;
                        ptx::mbar_arrive_expect_tx(&bars->full[st], (uint32_t)kPfBuf);
                        ptx::tma_load_3d(dst, map, &bars->full[st], 0, w.h, row, policy);
                        ptx::tma_load_3d(dst + kPfHalf, map, &bars->full[st], 64, w.h, row, policy);
                    }
                    __syncwarp();
                    ++x;
                };
                load_kv(0);
                // The queries' buffers are free once the item before has formed its last S.
                if (!stop && qloads > 0 && !pf_wait(&bars->q_empty, (qloads - 1) & 1, abort)) stop = true;
                if (stop) break;
                if (ptx::elect_one()) {
                    const uint32_t bytes = (uint32_t)(A.nq * A.g) * 128u;
                    ptx::mbar_arrive_expect_tx(&bars->q_full, 2u * bytes * (uint32_t)w.tiles);
                    for (int t = 0; t < w.tiles; ++t)
                        for (int c = 0; c < 2; ++c)
                            ptx::tma_load_3d(sQ + t * kPfBuf + c * kPfHalf, &A.qmap, &bars->q_full, c * 64, w.h * A.g,
                                             w.q0 + w.a + t * A.nq, policy);
                }
                __syncwarp();
                ++qloads;
                load_kv(1);
                if (!stop) hand_out(turn + 1);
                for (int y = 2; y < 2 * w.n && !stop; ++y) load_kv(y);
            }
            give_up();
            // Every issued copy lands before the CTA may exit.
            for (int y = max(x - kPfStages, 0); y < x; ++y)
                ptx::mbar_wait(&bars->full[y % kPfStages], (y / kPfStages) & 1, 50000000ull);
            if (qloads > 0) ptx::mbar_wait(&bars->q_full, (qloads - 1) & 1, 50000000ull);
        } else if (warp <= 10) {
            // -------------------------------------------------------- MMA, a warp for each tile
            // Few products queue up, and a wait, even one that is over, takes 60 cycles, in which the pipe
            // would run dry.  So the two warps take turns: one waits for what its tile needs while the other
            // issues.  A turn is not handed over before its products and their signals are issued: products of
            // two tiles in the queue delay both (8192 tokens: 409 us with three products left, 372 with the
            // signals left, 349 so; one warp for both tiles 375).
            const int t = warp - 9;
            const uint32_t idesc_s = pf_idesc<T>(false), idesc_o = pf_idesc<T>(true);
            const uint64_t qdesc = ptx::smem_desc_k_sw128(ptx::smem_u32(sQ)) + (uint32_t)(t * (kPfBuf >> 4));
            const uint64_t kdesc = ptx::smem_desc_k_sw128(ptx::smem_u32(ring));
            const uint64_t vdesc = smem_desc_mn_sw128(ptx::smem_u32(ring));
            const uint32_t dS = tmem + t * 128, dO = tmem + 256 + t * 128;
            auto wait = [&](uint64_t* bar, int phase) {
                if (!stop && !pf_wait(bar, phase & 1, abort)) stop = true;
                return !stop;
            };
            // The stage of a load and its parity, stepped.
            struct Place {
                int st = 0, parity = 0;
                __device__ __forceinline__ void step() {
                    if (++st == kPfStages) {
                        st = 0;
                        parity ^= 1;
                    }
                }
            };
            Place pk, pv;   // of the next K and V
            pv.step();
            int turns_taken = 0;
            // Stages as values that the compiler knows to be the warp's, so that descriptors stay in uniform registers.
            auto products_s = [&](int st) {   // S = Q K^T, K in stage st; one thread
                const uint64_t kd = kdesc + (uint32_t)(st * (kPfBuf >> 4));
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    const uint32_t ofs = (kk >> 2) * (kPfHalf >> 4) + (kk & 3) * 2;
                    ptx::mma_bf16(dS, qdesc + ofs, kd + ofs, idesc_s, kk > 0 ? 1u : 0u);
                }
            };
            auto products_o = [&](int st, bool add) {   // O += P V, V in stage st
                const uint64_t vd = vdesc + (uint32_t)(st * (kPfBuf >> 4));
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
                    mma_tmem_a(dO, dS + kk * 8, vd + kk * (2048 >> 4), idesc_o, add || kk > 0 ? 1u : 0u);
            };
            // A turn begins once the other tile's is over.
            auto begin_turn = [&]() {
                if (!wait(&bars->turn[t], t == 0 ? turns_taken + 1 : turns_taken)) return false;
                ++turns_taken;
                ptx::tc_fence_after();
                return true;
            };
            // The products of a block's V; a tile without rows only passes the stage on.  last: of the item.
            auto issue_o = [&](bool here, bool add, bool last) {
                const int st = ptx::warp_uniform(pv.st);
                if (ptx::elect_one()) {
                    if (here) {
                        products_o(st, add);
                        if (last) ptx::mma_commit(&bars->o_done[t]);
                        ptx::mma_commit(&bars->empty[st]);
                    } else {
                        ptx::mbar_arrive(&bars->empty[st]);
                    }
                }
                __syncwarp();
                pv.step();
                pv.step();
            };
            // Those of a K.  last: with the item's queries.
            auto issue_s = [&](bool here, bool last) {
                const int st = ptx::warp_uniform(pk.st);
                if (ptx::elect_one()) {
                    if (here) {
                        products_s(st);
                        ptx::mma_commit(&bars->s_full[t]);
                        ptx::mma_commit(&bars->empty[st]);
                        if (last) ptx::mma_commit(&bars->q_empty);
                    } else {
                        ptx::mbar_arrive(&bars->empty[st]);
                        if (last) ptx::mbar_arrive(&bars->q_empty);
                    }
                }
                __syncwarp();
                pk.step();
                pk.step();
            };
            auto end_turn = [&]() {
                if (ptx::elect_one()) ptx::mbar_arrive(&bars->turn[t ^ 1]);
                __syncwarp();
            };
            int qloads = 0, blocks = 0;   // blocks of this tile so far: the phase of its P
            Item w{}, next{};
            // One item further and no more where they are handed out: those behind one that sees nothing come once
            // the softmax warps have passed it, for which they may need the products that are still to be issued.
            auto next_item = [&]() {
                do {
                    if (!take_item(next)) return false;
                } while (!RAGGED && next.n == 0);
                return true;
            };
            auto sees = [&]() { return !RAGGED || next.n > 0; };
            auto wait_q = [&]() { return wait(&bars->full[pk.st], pk.parity) && wait(&bars->q_full, qloads++); };
            auto first_s = [&]() { issue_s(t < next.tiles, next.n == 1); };
            // The first S of the next item that sees a key, in a turn of its own.
            auto start = [&]() {
                do {
                    if (!next_item()) return false;
                } while (!sees());
                if (!wait_q() || !begin_turn()) return false;
                first_s();
                end_turn();
                return true;
            };
            bool more = start();
            while (more && !stop) {
                w = next;
                bool joined = false;   // the next item's first S goes behind this one's last products
                const bool here = t < w.tiles;
                const int n = w.n;
                for (int i = 0; i < n; ++i) {
                    const bool last = i + 1 == n;
                    if (last) {
                        more = next_item();
                        joined = more && sees();
                    }
                    if (stop || !wait(&bars->full[pv.st], pv.parity)) break;
                    if (w.edge(i) && !wait(&bars->clean[pv.st], pv.parity)) break;
                    if (!last && !wait(&bars->full[pk.st], pk.parity)) break;
                    if (last && joined && !wait_q()) break;
                    if (here && !wait(&bars->p_full[t], blocks++)) break;
                    if (here && !last) {   // most turns: nothing stands between the products
                        const int sv = ptx::warp_uniform(pv.st), sk = ptx::warp_uniform(pk.st);
                        if (!begin_turn()) break;
                        if (ptx::elect_one()) {
                            products_o(sv, i > 0);
                            ptx::mma_commit(&bars->empty[sv]);
                            products_s(sk);
                            ptx::mma_commit(&bars->s_full[t]);
                            ptx::mma_commit(&bars->empty[sk]);
                            if (i + 2 == n) ptx::mma_commit(&bars->q_empty);
                            ptx::mbar_arrive(&bars->turn[t ^ 1]);
                        }
                        __syncwarp();
                        pv.step();
                        pv.step();
                        pk.step();
                        pk.step();
                        continue;
                    }
                    if (!begin_turn()) break;
                    issue_o(here, i > 0, last);
                    if (!last) {
                        issue_s(here, i + 2 == n);
                    } else if (joined) {
                        first_s();
                    }
                    end_turn();
                }
                if (RAGGED && more && !joined) more = !stop && start();
            }
            give_up();
            // The products in flight end before TMEM is freed.
            if (ptx::elect_one()) ptx::mma_commit(&bars->mma_done);
            __syncwarp();
            ptx::mbar_wait(&bars->mma_done, 0, 50000000ull);
        } else {
            // -------------------------------------------------------- V blocks of partial sight
            // Every load is passed in turn: a parity says nothing of a stage several rounds ahead.
            Item w{};
            while (!stop && take_item(w)) {
                for (int y = 0; y < 2 * w.n; ++y, ++x) {
                    const int st = x % kPfStages;
                    if (!pf_wait(&bars->full[st], (x / kPfStages) & 1, abort)) {
                        stop = true;
                        break;
                    }
                    if ((y & 1) && w.edge(y >> 1)) {
                        // A look at eight vectors at once: their largest magnitude, NaN if there is one.
                        uint4* v = reinterpret_cast<uint4*>(ring + st * kPfBuf);
                        bool found = false;
#pragma unroll 2
                        for (int e0 = lane; e0 < kPfBuf / 16; e0 += 256) {
                            uint4 u[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) u[e] = v[e0 + 32 * e];
                            uint4 most = u[0];
#pragma unroll
                            for (int e = 1; e < 8; ++e)
                                most = make_uint4(largest<T>(most.x, u[e].x), largest<T>(most.y, u[e].y),
                                                  largest<T>(most.z, u[e].z), largest<T>(most.w, u[e].w));
                            if (!unbounded_mask<T>(largest<T>(largest<T>(most.x, most.y), largest<T>(most.z, most.w)))) continue;
                            found = true;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const uint4 m = make_uint4(unbounded_mask<T>(u[e].x), unbounded_mask<T>(u[e].y),
                                                           unbounded_mask<T>(u[e].z), unbounded_mask<T>(u[e].w));
                                v[e0 + 32 * e] = make_uint4(u[e].x & ~m.x, u[e].y & ~m.y, u[e].z & ~m.z, u[e].w & ~m.w);
                            }
                        }
                        if (found) bars->unbounded = 1;
                        ptx::fence_proxy_async_smem();
                    }
                    __syncwarp();
                    if (lane == 0) {
                        ptx::mbar_arrive(&bars->clean[st]);
                        ptx::mbar_arrive(&bars->empty[st]);
                    }
                }
            }
            give_up();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kPfSoftmaxRegs));
        // ------------------------------------------------------------ softmax
        const int t = warp >> 2, quad = warp & 3, row = quad * 32 + lane;
        const int row_q = row / A.g, j = row - row_q * A.g;
        const uint32_t lanes = (uint32_t)(quad * 32) << 16;
        const uint32_t tS = tmem + lanes + t * 128, tO = tmem + lanes + 256 + t * 128;
        const float sl2f = A.sl2;
        const uint64_t sl2 = ptx::pack_f32x2(sl2f, sl2f);
        // The infinities and NaN that a row sees in the blocks of partial sight: their weights
        // are positive, so each makes its output infinite or NaN.
        auto add_unbounded = [&](int p, int below, const Item& w, int n, auto add) {
#pragma unroll 1
            for (int i = 0; i < n; ++i) {
                if (!w.edge(i)) continue;
#pragma unroll 1
                for (int c = 0; c < kPfTile; ++c) {
                    const int key = w.block(i) * kPfTile + c;
                    if (key > p || (key <= below && key >= sinks)) continue;
                    const uint16_t* v = A.io.v + ((size_t)(w.k0 + key) * A.io.Hkv + w.h) * kHeadDim;
#pragma unroll 1
                    for (int d = 0; d < kHeadDim; ++d)
                        if (unbounded_mask<T>(v[d])) add(d, Half16<T>::unpack(v[d]).x);
                }
            }
        };
        int blocks = 0, outs = 0;   // blocks and items of this tile: the phases of its barriers
        Item w{};
        while (!stop && take_item(w)) {
            if (t >= w.tiles) continue;
            const int query = w.a + t * A.nq + row_q;
            const bool live = row < A.nq * A.g && query < w.b;        // the row is a real one
            const int p = w.off + query;
            const int below = A.io.window ? p - A.io.window : -1;     // keys up to here are out of the window
            const int n = w.n;
            float m = kNoLogit, l = 0.f;
            for (int i = 0; i < n; ++i, ++blocks) {
                if (!pf_wait(&bars->s_full[t], blocks & 1, abort)) {
                    stop = true;
                    break;
                }
                ptx::tc_fence_after();
                float s[128];
#pragma unroll
                for (int c = 0; c < 4; ++c) ptx::tmem_ld32(tS + c * 32, s + c * 32);
                ptx::tmem_wait_ld();
                if (w.edge(i)) {
                    // Bit c of the words: the row sees key t0 + c.  (Comparisons for each column
                    // became branches, 12,000 cycles a block.)
                    const int t0 = w.block(i) * kPfTile;
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int b0 = t0 + 32 * g;
                        const uint32_t seen = low_bits(p + 1 - b0) & (~low_bits(below + 1 - b0) | low_bits(sinks - b0));
#pragma unroll
                        for (int c = 0; c < 32; ++c) s[32 * g + c] = (seen >> c) & 1u ? s[32 * g + c] : -INFINITY;
                    }
                }
                // The weights of half the keys relative to m, as pairs of 16-bit values over S, and their sum.
                auto weights = [&](int c) {
                    const uint64_t ref = ptx::pack_f32x2(-m, -m);
                    uint64_t sum[4] = {0ull, 0ull, 0ull, 0ull};
                    uint32_t pk[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const uint64_t y = ptx::fma_f32x2(ptx::pack_f32x2(s[c * 64 + 2 * e], s[c * 64 + 2 * e + 1]), sl2, ref);
                        const float p0 = ptx::ex2(ptx::lo_f32(y)), p1 = ptx::ex2(ptx::hi_f32(y));
                        sum[e & 3] = ptx::add_f32x2(sum[e & 3], ptx::pack_f32x2(p0, p1));
                        pk[e] = Half16<T>::pack(p0, p1);
                    }
                    tmem_st32(tS + c * 32, pk);
                    const uint64_t all = ptx::add_f32x2(ptx::add_f32x2(sum[0], sum[1]), ptx::add_f32x2(sum[2], sum[3]));
                    return ptx::lo_f32(all) + ptx::hi_f32(all);
                };
                if (i == 0) {   // the row's first maximum
#pragma unroll
                    for (int e = 0; e < 128; e += 2) m = max3(m, s[e] * sl2f, s[e + 1] * sl2f);
                }
                float z = weights(0);
                z += weights(1);
                if (__any_sync(0xffffffffu, live && !(z < kMostWeight))) {
                    // The row's first logits, ones far above m, or NaN: m moves to the largest.
                    tmem_wait_st();   // these weights are written again
                    float mx = m;
#pragma unroll
                    for (int e = 0; e < 128; e += 2) mx = max3(mx, s[e] * sl2f, s[e + 1] * sl2f);
                    if (z < kMostWeight || !live) mx = m;
                    const float f = ptx::ex2(m - mx);
                    l *= f;
                    m = mx;
                    if (i > 0) {
                        // The outputs so far with it: the products of the block before were issued before
                        // this S, by the same thread, so that its signal covers them.
#pragma unroll 1
                        for (int d0 = 0; d0 < kHeadDim; d0 += 32) {
                            float o[32];
                            ptx::tmem_ld32(tO + d0, o);
                            ptx::tmem_wait_ld();
#pragma unroll
                            for (int d = 0; d < 32; ++d) o[d] *= f;
                            tmem_st32(tO + d0, reinterpret_cast<const uint32_t*>(o));
                        }
                    }
                    z = weights(0);
                    z += weights(1);
                }
                l += z;
                tmem_wait_st();
                ptx::tc_fence_before();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&bars->p_full[t]);
            }
            if (n > 0 && !stop && !pf_wait(&bars->o_done[t], outs++ & 1, abort)) stop = true;
            if (stop) break;
            ptx::tc_fence_after();
            const bool some = l > 0.f || l != l;
            const float inv = some ? 1.f / l : 0.f;
            const size_t at = (size_t)(w.q0 + query) * A.io.Hq + w.h * A.g + j;
            if constexpr (PARTS) {
                // Sums and maximum as they are, for prefill_join_kernel.
                const size_t prow = ((size_t)w.place * 2 + t) * kPfTile + row;
                float* dst = A.part_o + prow * kHeadDim;
#pragma unroll 1
                for (int c = 0; c < 4 && n > 0; ++c) {
                    float o[32];
                    ptx::tmem_ld32(tO + c * 32, o);
                    ptx::tmem_wait_ld();
                    if (live) {
#pragma unroll
                        for (int d = 0; d < 32; d += 8) st_global_v8(dst + c * 32 + d, reinterpret_cast<const uint32_t*>(o) + d);
                    }
                }
                ptx::tc_fence_before();
                if (live) {
                    A.part_ml[prow] = make_float2(n > 0 ? m : kNoLogit, l);
                    if (n > 0 && bars->unbounded) add_unbounded(p, below, w, n, [&](int d, float v) { dst[d] += v; });
                }
                __syncwarp();
                continue;
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float o[32];
                if (n > 0) {
                    ptx::tmem_ld32(tO + c * 32, o);
                    ptx::tmem_wait_ld();
                } else {
#pragma unroll
                    for (int d = 0; d < 32; ++d) o[d] = 0.f;
                }
#pragma unroll
                for (int d = 0; d < 32; ++d) o[d] = some ? o[d] * inv : 0.f;
                if (live) {
                    uint32_t u[16];
#pragma unroll
                    for (int d = 0; d < 16; ++d) u[d] = Half16<T>::pack(o[2 * d], o[2 * d + 1]);
                    st_global_v8(A.io.out + at * kHeadDim + c * 32, u);
                    st_global_v8(A.io.out + at * kHeadDim + c * 32 + 16, u + 8);
                }
            }
            ptx::tc_fence_before();   // O has been read before the next item's weights are handed over
            if (live && n > 0 && bars->unbounded) {
                uint16_t* dst = A.io.out + at * kHeadDim;
                add_unbounded(p, below, w, n, [&](int d, float v) {
                    dst[d] = (uint16_t)Half16<T>::pack(Half16<T>::unpack(dst[d]).x + v, 0.f);
                });
            }
            if (live && A.io.lse) A.io.lse[at] = some ? fmaf(m, 0.6931471805599453f, logf(l)) : -INFINITY;
            __syncwarp();
        }
        give_up();
    }
    __syncthreads();
    if (warp == 9) ptx::tmem_dealloc(tmem, kPfTmem);
}

// Rows whose blocks several items share: one warp a row, four dimensions a lane.
constexpr int kPjWarps = 8;
template <class T>
__global__ void __launch_bounds__(32 * kPjWarps) prefill_join_kernel(const __grid_constant__ PfArgs A) {
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    const int lane = threadIdx.x & 31, r = blockIdx.y * kPjWarps + (threadIdx.x >> 5);   // row of the pair
    const int first = blockIdx.x * A.parts, t = r / kPfTile, row = r % kPfTile;
    Item w{};
    const int query = row / A.g + t * A.nq;
    const int top = A.by_per.divide(blockIdx.x), sh = blockIdx.x - top * A.io.batch * A.io.Hkv, seq = A.by_heads.divide(sh);
    const bool live = make_item<true>(A, A.pairs - 1 - top, seq, Rows(A, seq), sh - seq * A.io.Hkv, 0, w) && row < A.nq * A.g && w.a + query < w.b;
    if (!live) return;
    auto prow = [&](int i) { return ((size_t)(first + i) * 2 + t) * kPfTile + row; };
    float M = kNoLogit, L = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < A.parts; ++i) M = fmaxf(M, A.part_ml[prow(i)].x);
    for (int i = 0; i < A.parts; ++i) {
        const float2 ml = A.part_ml[prow(i)];
        if (ml.x == kNoLogit && ml.y == 0.f) continue;   // a part that sees nothing wrote no sums
        const float f = ptx::ex2(ml.x - M);
        const float4 v = reinterpret_cast<const float4*>(A.part_o + prow(i) * kHeadDim)[lane];
        L = fmaf(f, ml.y, L);
        o = make_float4(fmaf(f, v.x, o.x), fmaf(f, v.y, o.y), fmaf(f, v.z, o.z), fmaf(f, v.w, o.w));
    }
    const bool some = L > 0.f || L != L;
    const float inv = some ? 1.f / L : 0.f;
    const size_t at = (size_t)(w.q0 + w.a + query) * A.io.Hq + w.h * A.g + row % A.g;
    reinterpret_cast<uint2*>(A.io.out + at * kHeadDim)[lane] =
        some ? make_uint2(Half16<T>::pack(o.x * inv, o.y * inv), Half16<T>::pack(o.z * inv, o.w * inv)) : make_uint2(0u, 0u);
    if (lane == 0 && A.io.lse) A.io.lse[at] = some ? fmaf(M, 0.6931471805599453f, logf(L)) : -INFINITY;
}

template <class T>
cudaError_t launch_typed(const PfArgs& a, long long used_pairs, int num_sms, cudaStream_t st) {
    const dim3 grid((unsigned)std::min(a.items, num_sms));
    // Places that shorter sequences leave unused make the shares uneven, unless the turns are many, while an
    // item that is handed over costs half a microsecond more.  Shared out by place and by item, us: 8192 and 5001 tokens 503 and 465 (14
    // turns), one of 8192 and four of 100 391 and 333 (34), 24 of 100 to 1000 133 and 116 (20); but 32 of 1000
    // 289 and 308 (nothing unused), 32 of 1 to 4000 1064 and 1080 (106 turns).
    const bool ragged = (long long)a.pairs * a.io.batch * 15 > used_pairs * 16 && a.items <= 64 * num_sms;
    if (a.parts == 1)
        return ragged
                   ? launch_prio(prefill_kernel<T, false, true>, grid, dim3(kPfThreads), kPfSmem, st, 0, true, a)
                   : launch_prio(prefill_kernel<T, false, false>, grid, dim3(kPfThreads), kPfSmem, st, 0, true, a);
    cudaError_t e = launch_prio(prefill_kernel<T, true, false>, grid, dim3(kPfThreads), kPfSmem, st, 0, true, a);
    if (e != cudaSuccess) return e;
    return launch_prio(prefill_join_kernel<T>, dim3((unsigned)(a.items / a.parts), 2 * kPfTile / kPjWarps), dim3(32 * kPjWarps),
                       0, st, 0, true, a);
}

// Pairs of tiles over all sequences, and the parts that each pair's blocks are divided into: as
// many as SMs would be idle otherwise, of two blocks and more.
int split_parts(const PrefillPlan& p, int num_sms) {
    const long long whole = (long long)p.pairs * p.batch * p.Hkv;
    return (int)std::max<long long>(1, std::min<long long>(num_sms / std::max<long long>(whole, 1), p.max_blocks / 2));
}

}  // namespace

cudaError_t configure_prefill() {
    cudaError_t e = cudaSuccess;
    auto one = [&](auto kernel) {
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPfSmem);
    };
    one(prefill_kernel<__nv_bfloat16, false, false>);
    one(prefill_kernel<__nv_bfloat16, false, true>);
    one(prefill_kernel<__nv_bfloat16, true, false>);
    one(prefill_kernel<__half, false, false>);
    one(prefill_kernel<__half, false, true>);
    one(prefill_kernel<__half, true, false>);
    return e;
}

PrefillPlan plan_prefill(int batch, int Hq, int Hkv, int max_q, int max_k, int window, int sinks, int num_sms) {
    PrefillPlan p{};
    p.batch = batch;
    p.Hkv = Hkv;
    p.nq = kPfTile / (Hq / Hkv);
    p.pairs = (max_q + 2 * p.nq - 1) / (2 * p.nq);
    long long blocks = (max_k + kPfTile - 1) / kPfTile;
    // A window's blocks, and those of the first tokens.
    if (window)
        blocks = std::min(blocks, ((long long)window + 2 * p.nq) / kPfTile + 2 + ((long long)std::min(sinks, max_k) + kPfTile - 1) / kPfTile);
    p.max_blocks = (int)blocks;
    p.parts = split_parts(p, num_sms);
    const size_t items = (size_t)p.pairs * batch * Hkv * p.parts;
    p.scratch = p.parts > 1 ? items * 2 * kPfTile * (kHeadDim * sizeof(float) + sizeof(float2)) : 0;
    return p;
}

cudaError_t launch_prefill(const PrefillIO& io, const PrefillPlan& plan, int num_sms, cudaStream_t st) {
    PfArgs a{};
    a.io = io;
    a.g = io.Hq / io.Hkv;
    a.nq = plan.nq;
    a.pairs = plan.pairs;
    a.parts = plan.parts;
    const long long items = (long long)a.pairs * io.batch * io.Hkv * a.parts;
    if (items > 0x3fffffffll) return cudaErrorInvalidConfiguration;
    a.items = (int)items;
    a.part_o = static_cast<float*>(io.scratch);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + (size_t)items * 2 * kPfTile * kHeadDim);
    a.by_per.set(io.batch * io.Hkv);
    a.by_heads.set(io.Hkv);
    a.sl2 = io.scale * 1.4426950408889634f;
    a.fault = test_fault() == 4 ? 1 : 0;
    const uint64_t row = (uint64_t)kHeadDim * 2;
    const uint64_t qd[3] = {(uint64_t)kHeadDim, (uint64_t)io.Hq, (uint64_t)io.total_q}, qs[2] = {row, row * io.Hq};
    const uint32_t qb[3] = {64, (uint32_t)a.g, (uint32_t)a.nq};
    // Without any key nothing is loaded by the maps of K and V.
    const bool keys = io.total_k > 0;
    const uint64_t kd[3] = {(uint64_t)kHeadDim, (uint64_t)io.Hkv, (uint64_t)std::max(io.total_k, 1)}, ks[2] = {row, row * io.Hkv};
    const uint32_t kb[3] = {64, 1, (uint32_t)kPfTile};
    cudaError_t e = encode_tensor_map(&a.qmap, io.dtype, 3, io.q, qd, qs, qb);
    if (e == cudaSuccess) e = encode_tensor_map(&a.kmap, io.dtype, 3, keys ? io.k : io.q, kd, ks, kb);
    if (e == cudaSuccess) e = encode_tensor_map(&a.vmap, io.dtype, 3, keys ? io.v : io.q, kd, ks, kb);
    if (e != cudaSuccess) return e;
    return io.dtype == 1 ? launch_typed<__half>(a, plan.used_pairs, num_sms, st) : launch_typed<__nv_bfloat16>(a, plan.used_pairs, num_sms, st);
}

}  // namespace kvec
