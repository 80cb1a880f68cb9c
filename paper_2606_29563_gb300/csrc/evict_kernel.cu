// Eviction from the paged cache by accumulated attention weight.  Of a KV head's n slots
// the first `sinks`, the last `recent` and the best of the others by weight stay, `budget`
// in all; their rows are copied in ascending order to new pages.
//
// Two launches.  evict_select_kernel ranks a (sequence, KV head) row in a block: the keys
// in registers and one histogram over their own range (hist_select.cuh) for rows up to
// 32768, a radix select that sweeps the row in L2 for longer ones; it writes the kept
// slots.  evict_copy_kernel moves the rows, one half-warp a row of K and of V: HBM-bound,
// and spread over the device whatever the number of rows (the new pages are none of the
// old, so no copy waits for another).  One launch of clusters whose first CTA ranks while the
// others wait was slower from 32 rows on: the waiting CTAs hold the SMs.
//
// Measured, in us (in brackets the bytes at the measured copy rate): 8 rows of 576 slots to
// 512 7.1 (0.6), the chain of two launches and six barriers; 128 rows of 1000 to 4096 slots to
// 1024 29.3 (20.2); 512 of 2100 to 2048 175 (161); 8 of 32768 to 8192 27 (10.2), of 65536, by
// sweeps, 65 to 74 (10.3), of 131072 130 (10.6).  The kernel goes by the bound on the lengths: 8 rows of
// 576 slots take 7.4 under their own, 13.5 under one of 32768 and 8.5 under one of 131072 (by sweeps).
// Small blocks of few rows fill the device best: two rows of K and V in flight a half-warp and
// 128 threads 29.3, four and 256 31.0, eight and 256 36.6.
#include "hist_select.cuh"
#include "kvec_internal.cuh"

namespace kvec {

namespace {

struct EvictArgs {
    EvictIO io;
    PagedCacheView c;
};

__device__ __forceinline__ int clamped_len(const EvictArgs& A, int s) {
    return min(max(__ldg(&A.c.lens[s]), 0), A.io.max_len);
}

// Row of slot `slot` of KV head h in the pages of `table`; -1 on no page.
__device__ __forceinline__ long long slot_row(const int* table, int slot, int h, int Hkv, const PagedCacheView& c) {
    const int page = __ldg(&table[slot >> c.log_page]);
    if (page < 0 || page >= c.num_pages) return -1;
    return (((long long)page * Hkv + h) << c.log_page) + (slot & ((1 << c.log_page) - 1));
}

// Ranking key of a weight, > 0: -0 ranks as 0, NaN as minus infinity.
__device__ __forceinline__ uint32_t weight_key(float w) {
    return float_order_key(w != w ? -INFINITY : w + 0.f);
}

// The slots of bits[] (one bit a slot, nwords words) to kept[0 ..], ascending, and -1
// behind them up to budget.
template <int NT>
__device__ void write_kept(const uint32_t* bits, int nwords, int* kept, int budget, int* wsum) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int kWarps = NT / 32;
    const int per = (nwords + kWarps - 1) / kWarps;   // words of a warp, contiguous
    const int w0 = min(warp * per, nwords), w1 = min(w0 + per, nwords);
    int c = 0;
    for (int w = w0 + lane; w < w1; w += 32) c += __popc(bits[w]);
    c = __reduce_add_sync(0xffffffffu, c);
    if (lane == 0) wsum[warp] = c;
    __syncthreads();
    int before = lane < warp && lane < kWarps ? wsum[lane] : 0;
    before = __reduce_add_sync(0xffffffffu, before);
    int total = lane < kWarps ? wsum[lane] : 0;
    total = __reduce_add_sync(0xffffffffu, total);
    for (int w = w0; w < w1; ++w) {
        const uint32_t b = bits[w];
        if ((b >> lane) & 1u) kept[before + __popc(b & ((1u << lane) - 1u))] = w * 32 + lane;
        before += __popc(b);
    }
    for (int j = total + tid; j < budget; j += NT) kept[j] = -1;
}

// Rows of up to NT * KPT slots.
template <int NT, int KPT>
__global__ void __launch_bounds__(NT) evict_select_kernel(const __grid_constant__ EvictArgs A) {
    using HS = HistSelect<NT, KPT>;
    __shared__ HistSelectShared sm;
    __shared__ __align__(16) uint32_t bits[HS::kWords];
    __shared__ int wsum[32];
    const int h = blockIdx.x, s = blockIdx.y, tid = threadIdx.x;
    HS::clear(sm);
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    const int n = clamped_len(A, s), B = A.io.budget, Hkv = A.io.Hkv;
    int* kept = A.io.kept + ((size_t)s * Hkv + h) * B;
    const int* table = A.c.table + (size_t)s * A.c.max_pages;
    // The weights of every slot that there may be: their pages do not wait for the length.
    float4 w[KPT / 4];
#pragma unroll
    for (int g = 0; g < KPT / 4; ++g) {
        const int j = HS::position(4 * g);   // four slots of one page
        w[g] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        if (j < A.io.max_len) {
            const long long row = slot_row(table, j, h, Hkv, A.c);
            if (row >= 0) w[g] = *reinterpret_cast<const float4*>(A.c.weights + row);
        }
    }
    if (h == 0 && tid == 0) A.io.new_lens[s] = min(n, B);
    if (n <= B) {
        for (int j = tid; j < B; j += NT) kept[j] = j < n ? j : -1;
        return;
    }
    const int lo = A.io.sinks, hi = n - A.io.recent;   // the ranked slots; sinks + recent <= B < n
    uint32_t key[KPT];
#pragma unroll
    for (int g = 0; g < KPT / 4; ++g) {
        const int j = HS::position(4 * g);
        const float v[4] = {w[g].x, w[g].y, w[g].z, w[g].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) key[4 * g + e] = j + e >= lo && j + e < hi ? weight_key(v[e]) : 0u;
    }
    HS hs{sm, B - A.io.sinks - A.io.recent};
    __syncthreads();   // clear()
    uint32_t match = 0u, sel = 0u;
    if (hs.k > 0) sel = hs.begin(key, match);
    // The slots that are always kept.
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const int j = HS::position(i);
        if (j < lo || (j >= hi && j < n)) sel |= 1u << i;
    }
    HS::store(sel, bits);
    __syncthreads();
    if (hs.k > 0) hs.finish(key, match, bits);
    __syncthreads();
    write_kept<NT>(bits, (n + 31) >> 5, kept, B, wsum);
}

// Rows of any length: the key of rank k by its digits (12, 12 and 8 bits), one sweep of the
// row for each, then the kept slots in order, the lowest of the equal keys first.
constexpr int kSweepThreads = 1024;
__global__ void __launch_bounds__(kSweepThreads) evict_sweep_kernel(const __grid_constant__ EvictArgs A) {
    __shared__ uint32_t hist[4096];
    __shared__ int wsum[32], wsum2[32];
    __shared__ int sdigit, sabove;
    const int h = blockIdx.x, s = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    const int n = clamped_len(A, s), B = A.io.budget, Hkv = A.io.Hkv;
    int* kept = A.io.kept + ((size_t)s * Hkv + h) * B;
    if (h == 0 && tid == 0) A.io.new_lens[s] = min(n, B);
    if (n <= B) {
        for (int j = tid; j < B; j += kSweepThreads) kept[j] = j < n ? j : -1;
        return;
    }
    const int lo = A.io.sinks, hi = n - A.io.recent;
    const int* table = A.c.table + (size_t)s * A.c.max_pages;
    // The keys of four consecutive slots, 0 for those that are not ranked.
    auto load4 = [&](int j, uint32_t (&key)[4]) {
        float4 w = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        if (j < n) {
            const long long row = slot_row(table, j, h, Hkv, A.c);
            if (row >= 0) w = *reinterpret_cast<const float4*>(A.c.weights + row);
        }
        const float v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) key[e] = j + e >= lo && j + e < hi ? weight_key(v[e]) : 0u;
    };
    const int k = B - A.io.sinks - A.io.recent;
    uint32_t prefix = 0u;   // the digits found
    int left = k;           // keys to take among those that share them
    int shift = 32;
    while (k > 0 && shift > 0) {
        const int bits = min(12, shift), top = shift;
        shift -= bits;
        for (int i = tid; i < 4096; i += kSweepThreads) hist[i] = 0u;
        __syncthreads();
        for (int j = tid * 4; j < n; j += kSweepThreads * 4) {
            uint32_t key[4];
            load4(j, key);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (key[e] != 0u && (top == 32 || (key[e] >> top) == prefix))
                    atomicAdd(&hist[(key[e] >> shift) & ((1u << bits) - 1u)], 1u);
        }
        __syncthreads();
        // Thread t: bins 4095 - 4 t down to 4092 - 4 t.
        int own = 0;
        uint32_t c[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) own += (int)(c[b] = hist[4095 - 4 * tid - b]);
        int incl = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        if (lane == 31) wsum[warp] = incl;
        __syncthreads();
        int before = lane < warp ? wsum[lane] : 0;
        before = __reduce_add_sync(0xffffffffu, before) + incl - own;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            if (before < left && left <= before + (int)c[b]) {
                sdigit = 4095 - 4 * tid - b;
                sabove = before;
            }
            before += (int)c[b];
        }
        __syncthreads();
        prefix = (prefix << bits) | (uint32_t)sdigit;
        left -= sabove;
        __syncthreads();   // before the next sweep's writes
    }
    // Every key above `prefix` and the first `left` equal ones.
    int out = 0, equal = 0;   // slots written, equal keys met
    for (int j0 = 0; j0 < n; j0 += kSweepThreads * 4) {
        const int j = j0 + tid * 4;
        uint32_t key[4];
        load4(j, key);
        int eq = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) eq += k > 0 && key[e] == prefix ? 1 : 0;
        int ie = eq;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, ie, o);
            if (lane >= o) ie += y;
        }
        if (lane == 31) wsum[warp] = ie;
        __syncthreads();
        int rank = equal + ie - eq + __reduce_add_sync(0xffffffffu, lane < warp ? wsum[lane] : 0);
        equal += __reduce_add_sync(0xffffffffu, wsum[lane]);
        uint32_t take = 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool always = j + e < lo || (j + e >= hi && j + e < n);
            const bool same = k > 0 && key[e] == prefix;
            if (always || (k > 0 && key[e] > prefix) || (same && rank < left)) take |= 1u << e;
            rank += same ? 1 : 0;
        }
        const int c = __popc(take);
        int ic = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, ic, o);
            if (lane >= o) ic += y;
        }
        if (lane == 31) wsum2[warp] = ic;
        __syncthreads();
        int at = out + ic - c + __reduce_add_sync(0xffffffffu, lane < warp ? wsum2[lane] : 0);
        out += __reduce_add_sync(0xffffffffu, wsum2[lane]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if ((take >> e) & 1u) kept[at++] = j + e;
        __syncthreads();   // the sums are read before the next sweep's
    }
}

constexpr int kCopyThreads = 128;
constexpr int kCopyPer = 2;                                   // rows of a half-warp
constexpr int kCopyRows = kCopyThreads / 16 * kCopyPer;       // rows of a block

__global__ void __launch_bounds__(kCopyThreads) evict_copy_kernel(const __grid_constant__ EvictArgs A) {
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    const int h = blockIdx.y, s = blockIdx.z, l16 = threadIdx.x & 15, Hkv = A.io.Hkv, B = A.io.budget;
    const int most = min(A.io.max_len, B);
    const int j0 = blockIdx.x * kCopyRows + (threadIdx.x >> 4);
    const int* kept = A.io.kept + ((size_t)s * Hkv + h) * B;
    const int* table = A.c.table + (size_t)s * A.c.max_pages;
    const int* fresh = A.io.new_table + (size_t)s * A.io.new_max_pages;
    long long src[kCopyPer], dst[kCopyPer];
#pragma unroll
    for (int i = 0; i < kCopyPer; ++i) {
        const int j = j0 + i * (kCopyThreads / 16);
        src[i] = dst[i] = -1;
        const int from = j < most ? kept[j] : -1;   // -1 past the kept ones
        if (from >= 0) {
            src[i] = slot_row(table, from, h, Hkv, A.c);
            dst[i] = slot_row(fresh, j, h, Hkv, A.c);
        }
    }
    uint4 k[kCopyPer], v[kCopyPer];
    float w[kCopyPer];
#pragma unroll
    for (int i = 0; i < kCopyPer; ++i) {
        if (src[i] < 0 || dst[i] < 0) continue;
        k[i] = reinterpret_cast<const uint4*>(A.c.k + src[i] * kHeadDim)[l16];
        v[i] = reinterpret_cast<const uint4*>(A.c.v + src[i] * kHeadDim)[l16];
        if (l16 == 0) w[i] = A.c.weights[src[i]];
    }
#pragma unroll
    for (int i = 0; i < kCopyPer; ++i) {
        if (src[i] < 0 || dst[i] < 0) continue;
        reinterpret_cast<uint4*>(A.c.k + dst[i] * kHeadDim)[l16] = k[i];
        reinterpret_cast<uint4*>(A.c.v + dst[i] * kHeadDim)[l16] = v[i];
        if (l16 == 0) A.c.weights[dst[i]] = w[i];
    }
}

}  // namespace

cudaError_t launch_evict(const EvictIO& io, const PagedCacheView& c, cudaStream_t st) {
    const EvictArgs a{io, c};
    const dim3 rows((unsigned)io.Hkv, (unsigned)io.batch);
    cudaError_t e;
    if (io.max_len <= 4096)
        e = launch_prio(evict_select_kernel<256, 16>, rows, dim3(256), 0, st, 0, true, a);
    else if (io.max_len <= 8192)
        e = launch_prio(evict_select_kernel<512, 16>, rows, dim3(512), 0, st, 0, true, a);
    else if (io.max_len <= 16384)
        e = launch_prio(evict_select_kernel<1024, 16>, rows, dim3(1024), 0, st, 0, true, a);
    else if (io.max_len <= kMaxRegisterRow)
        e = launch_prio(evict_select_kernel<1024, 32>, rows, dim3(1024), 0, st, 0, true, a);
    else
        e = launch_prio(evict_sweep_kernel, rows, dim3(kSweepThreads), 0, st, 0, true, a);
    if (e != cudaSuccess) return e;
    const int most = io.budget < io.max_len ? io.budget : io.max_len;
    const dim3 grid((unsigned)((most + kCopyRows - 1) / kCopyRows), (unsigned)io.Hkv, (unsigned)io.batch);
    return launch_prio(evict_copy_kernel, grid, dim3(kCopyThreads), 0, st, 0, true, a);
}

}  // namespace kvec
