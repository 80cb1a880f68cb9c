// Queries, keys and values of new tokens made ready for attention: the norm of every
// query and key head, the rotation by position, and the store into the paged cache.
// For a row x of 128 values, in fp32:
//   y = x * rsqrt(mean(x^2) + eps) * w,   (a, b) -> (a c - b s, b c + a s) per pair.
//
// A half-warp owns a head's row, eight values (16 bytes) a lane; the sum of squares and
// the partner values of the half-split pairs come by shuffles.  A block takes a token's rows
// together, so that the position's cosines and sines are loaded once for all of them, and in
// a prefill several tokens one after the other: where they belong (position, sequence, page) is
// found at the start by a thread a token, not in a chain of loads before each.
//
// HBM-bound: 82676 tokens of 32 + 2 x 8 heads (2.07 GB) in 333 us, 6.2 TB/s, 92 % of the
// measured copy rate (registers bounded to 64, so that eight blocks are resident: with 80 and
// one token a block 556 us).  One token 2.3 us, the launch.  Between: 1600 tokens 9.9 us for 5.9 of bytes, 3200
// 20.0 (11.8), 6400 32.9 (23.7), 12800 59 (47), as a block's chain of look-ups (sequence, position, length,
// page) and its table row come before each one or two tokens' rows.
#include "half_types.cuh"
#include "kvec_internal.cuh"

namespace kvec {

namespace {

constexpr int kRotWarps = 4;                  // warps of a block, two rows each at a time
constexpr int kRotRows = 2 * kRotWarps;

struct RotateArgs {
    RotateIO io;
    PagedCacheView c;
    int heads;           // Hq + 2 Hkv, or Hq + Hkv without values
};

__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

template <class T>
__device__ __forceinline__ void unpack8(const uint4& w, float (&v)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = Half16<T>::unpack(u[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}

// A token's position (-1: padding, nothing is written) and its row of KV head 0 in the pages
// (-1: none).
struct Place {
    long long row;
    int pos;
};

__device__ __forceinline__ Place place_of(const RotateArgs& A, int t) {
    const RotateIO& io = A.io;
    Place p{-1, io.positions[t]};
    if (p.pos < 0 || p.pos >= io.max_positions) p.pos = -1;
    int s = t, left = 1;
    if (io.cu) {
        // The last sequence that starts at or before t.
        int lo = 0, hi = io.batch;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (__ldg(&io.cu[mid]) <= t) lo = mid; else hi = mid - 1;
        }
        s = lo;
        if (s < io.batch) left = __ldg(&io.cu[s + 1]) - t;
    }
    if (s >= io.batch) p.pos = -1;       // behind the last sequence
    if (A.c.k && p.pos >= 0) {
        const long long at = (long long)__ldg(&A.c.lens[s]) - left;
        if (at >= 0 && at < A.c.capacity) {
            const int slot = (int)at;
            const int page = __ldg(&A.c.table[(size_t)s * A.c.max_pages + (slot >> A.c.log_page)]);
            if (page >= 0 && page < A.c.num_pages)
                p.row = ((long long)page * io.Hkv << A.c.log_page) + (slot & ((1 << A.c.log_page) - 1));
        }
    }
    return p;
}

// NR: rows of a token that a half-warp takes, NT: tokens of a block.  IL: interleaved pairs.
template <class T, int NR, int NT, bool IL>
__global__ void __launch_bounds__(32 * kRotWarps, 8) rotate_kernel(const __grid_constant__ RotateArgs A) {
    __shared__ Place places[NT];
    const int lane = threadIdx.x & 31, l16 = lane & 15;
    const int t0 = blockIdx.x * NT, u0 = blockIdx.y * (kRotRows * NR) + (threadIdx.x >> 4);
    asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    const RotateIO& io = A.io;
    const int Hq = io.Hq, Hkv = io.Hkv, heads = A.heads;
    const int rot = io.rot_dim, half = rot >> 1;
    const bool turn = l16 * 8 < rot, second = !IL && l16 * 8 >= half;
    const int partner = turn && !IL ? (lane & 16) | (second ? l16 - (rot >> 4) : l16 + (rot >> 4)) : lane;
    const int nt = min(NT, io.num_tokens - t0);
    if constexpr (NT > 1) {
        if (threadIdx.x < nt) places[threadIdx.x] = place_of(A, t0 + threadIdx.x);
        __syncthreads();
    }
#pragma unroll 1
    for (int k = 0; k < nt; ++k) {
        const int t = t0 + k;
        // Plain loads: an output may lie over its input, each row read before it is written.
        uint4 x[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int u = u0 + i * kRotRows;
            x[i] = make_uint4(0u, 0u, 0u, 0u);
            if (u >= heads) continue;
            const uint16_t* row = u < Hq         ? io.q + (size_t)t * io.q_stride + (size_t)u * kHeadDim
                                  : u < Hq + Hkv ? io.k + (size_t)t * io.k_stride + (size_t)(u - Hq) * kHeadDim
                                                 : io.v + (size_t)t * io.v_stride + (size_t)(u - Hq - Hkv) * kHeadDim;
            x[i] = *reinterpret_cast<const uint4*>(row + l16 * 8);
        }
        const Place at = NT > 1 ? places[k] : place_of(A, t);
        if (at.pos < 0) continue;
        float c[8], s[8];
        if (turn) {
            const float* tab = io.rot_table + (size_t)at.pos * rot;
            if constexpr (IL) {
                const float4 a = __ldg(reinterpret_cast<const float4*>(tab + l16 * 4));
                const float4 b = __ldg(reinterpret_cast<const float4*>(tab + half + l16 * 4));
                c[0] = a.x; c[1] = a.y; c[2] = a.z; c[3] = a.w;
                s[0] = b.x; s[1] = b.y; s[2] = b.z; s[3] = b.w;
            } else {
                load8(tab + l16 * 8 - (second ? half : 0), c);
                load8(tab + half + l16 * 8 - (second ? half : 0), s);
                // (a, b) -> (a c - b s, b c + a s): the second of a pair adds.
                if (!second) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e] = -s[e];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int u = u0 + i * kRotRows;
            const bool isq = u < Hq, isk = !isq && u < Hq + Hkv;
            uint4 out = x[i];   // a value row is copied as it is
            // The half-warps of a warp share the shuffles: both stay, whatever they store.
            if (__any_sync(0xffffffffu, isq || isk)) {
                float y[8];
                unpack8<T>(x[i], y);
                const uint16_t* norm = isq ? io.q_norm : isk ? io.k_norm : nullptr;
                if (io.q_norm || io.k_norm) {
                    float sq = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sq = fmaf(y[e], y[e], sq);
#pragma unroll
                    for (int o = 8; o; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
                    if (norm) {
                        const float r = rsqrtf(fmaf(sq, 1.f / kHeadDim, io.eps));
                        float w[8];
                        unpack8<T>(__ldg(reinterpret_cast<const uint4*>(norm) + l16), w);
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] *= r * w[e];
                    }
                }
                if constexpr (IL) {
                    if (turn) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float a = y[2 * e], b = y[2 * e + 1];
                            y[2 * e] = a * c[e] - b * s[e];
                            y[2 * e + 1] = b * c[e] + a * s[e];
                        }
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float z = __shfl_sync(0xffffffffu, y[e], partner);
                        if (turn) y[e] = y[e] * c[e] + z * s[e];
                    }
                }
                if (isq || isk)
                    out = make_uint4(Half16<T>::pack(y[0], y[1]), Half16<T>::pack(y[2], y[3]), Half16<T>::pack(y[4], y[5]),
                                     Half16<T>::pack(y[6], y[7]));
            }
            if (u >= heads) continue;
            if (isq) {
                reinterpret_cast<uint4*>(io.q_out + ((size_t)t * Hq + u) * kHeadDim)[l16] = out;
                continue;
            }
            const int h = isk ? u - Hq : u - Hq - Hkv;
            if (isk && io.k_out) reinterpret_cast<uint4*>(io.k_out + ((size_t)t * Hkv + h) * kHeadDim)[l16] = out;
            if (at.row < 0) continue;
            const size_t row = (size_t)at.row + ((size_t)h << A.c.log_page);
            reinterpret_cast<uint4*>((isk ? A.c.k : A.c.v) + row * kHeadDim)[l16] = out;
            if (isk && A.c.weights && l16 == 0) A.c.weights[row] = 0.f;
        }
    }
}

template <class T, int NR, int NT>
cudaError_t launch_rows(const RotateArgs& a, cudaStream_t st) {
    const dim3 grid((unsigned)((a.io.num_tokens + NT - 1) / NT), (unsigned)((a.heads + kRotRows * NR - 1) / (kRotRows * NR)));
    if (a.io.interleaved) return launch_prio(rotate_kernel<T, NR, NT, true>, grid, dim3(32 * kRotWarps), 0, st, 0, true, a);
    return launch_prio(rotate_kernel<T, NR, NT, false>, grid, dim3(32 * kRotWarps), 0, st, 0, true, a);
}

template <class T>
cudaError_t launch_typed(const RotateArgs& a, cudaStream_t st) {
    // By the rows of the call (tokens x heads).  Few are best all in flight at once, a row a
    // half-warp; many share their tokens' tables and places.  Measured with 48 heads, norms and
    // a cache, in us: 200 tokens 3.7 (three rows a half-warp 3.8), 400 5.2 (4.6); 1600 9.7
    // (six rows, two tokens 11.7), 3200 17.4 (17.2), 6400 37.5 (32.5; four tokens 36.0); 12800
    // tokens two 59.1, four 58.9; 82676 346 and 333.
    const long long rows = (long long)a.io.num_tokens * a.heads;
    if (rows <= 12000) return launch_rows<T, 1, 1>(a, st);
    if (rows <= 150000) return launch_rows<T, 3, 1>(a, st);
    if (rows <= 600000) return launch_rows<T, 6, 2>(a, st);
    return launch_rows<T, 6, 4>(a, st);
}

}  // namespace

cudaError_t launch_rotate(const RotateIO& io, const PagedCacheView& c, cudaStream_t st) {
    RotateArgs a{io, c, io.Hq + (c.k ? 2 : 1) * io.Hkv};
    return io.dtype == 1 ? launch_typed<__half>(a, st) : launch_typed<__nv_bfloat16>(a, st);
}

}  // namespace kvec
