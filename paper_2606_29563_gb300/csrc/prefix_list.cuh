// The work on prefixes that groups of sequences share: the 128-key blocks of all (group, KV head, pair of 128-row tiles)
// items, how the CTAs of prefill_kernel's PAGED form share them, and where these leave the sums that
// shared_join_kernel reads.
#pragma once

#include "kvec_internal.cuh"

namespace kvec {

constexpr int kPrefixTile = 128;   // rows of a tile, keys of a block

// What group r of sequences shares: its sequences [q0, q0 + n), the keys of its prefix and their blocks.
struct PrefixGroup {
    int q0, n, len, nb, pairs;
    __device__ __forceinline__ PrefixGroup(const PrefixGeom& A, int r) : q0(0), n(0), len(0), nb(0), pairs(0) {
        if (r >= A.groups) return;
        const int batch = A.batch;
        q0 = min(max(__ldg(&A.cu[r]), 0), batch);
        n = max(min(max(__ldg(&A.cu[r + 1]), 0), batch) - q0, 0);
        len = min(max(__ldg(&A.lens[r]), 0), A.max_prefix);
        nb = (len + kPrefixTile - 1) / kPrefixTile;
        pairs = (n + 2 * A.nq - 1) / (2 * A.nq);
    }
    // Places of an item in the list of all blocks: ahead of its blocks stand some for what beginning and ending it takes.
    static constexpr int kCost = 1;
    __device__ __forceinline__ int places() const { return nb && pairs ? nb + kCost : 0; }
    // Row of the sums that an item's CTAs leave: this for the first query of its pair, and 2 kPrefixTile rows further on for
    // each CTA before the one that leaves them (so that no two are in each other's way: from a CTA's item to its next
    // this grows by the rows of the first, and an item that goes on in the next CTA has 2 kPrefixTile rows at most).
    __device__ __forceinline__ int first_row(const PrefixGeom& A, int h, int pair) const {
        return q0 * A.Hq + (h * n + pair * 2 * A.nq) * A.g;
    }
};

// The sum of f over [from, to), by a whole warp: a lane each 32nd where there are more than a few.  (Up to 2048 are asked for
// for each sequence: 8192 sequences in as many groups take 719 us, and 1762 with one after the other by every lane.)
template <class F>
__device__ __forceinline__ long long sum_by_lanes(int from, int to, F f) {
    long long sum = 0;
    if (to - from <= 4) {
        for (int k = from; k < to; ++k) sum += f(k);
        return sum;
    }
    for (int k = from + (int)(threadIdx.x & 31); k < to; k += 32) sum += f(k);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return sum;
}

// How the CTAs share the work, as a warp sees it: lane l holds the groups l * per .. l * per + per - 1.
//
// If no item's blocks need to be cut into chunks much shorter than the mean share (a fourth above it at most), and there
// are CTAs enough, CTA c takes chunk c of them in the order (group, head, chunk, pair): the pairs of a group and head read the
// same keys and values at the same time, which then come from memory once.  Else the CTAs take even shares of the list of
// all items' blocks (longest = 0).  Three groups of 101, 42 and 17 sequences behind 32768, 8001 and 20000 slots: 140.4 us by
// chunks (251 MB read for the prefixes), 142.3 by shares (401 MB); four sequences behind 500 slots 14.3 and 18.1.
struct GroupList {
    int per, longest;                // blocks of a chunk at most
    long long before, mine, total;   // chunks or places: of the lanes before, of this lane, of all
    __device__ __forceinline__ static int chunks(const PrefixGroup& gr, int longest) {
        return gr.pairs ? (gr.nb + longest - 1) / longest : 0;
    }
    // Chunks or places of a group.
    __device__ __forceinline__ long long part(const PrefixGeom& A, const PrefixGroup& gr) const {
        return (long long)(longest ? chunks(gr, longest) : gr.places()) * gr.pairs * A.Hkv;
    }
    __device__ __forceinline__ GroupList(const PrefixGeom& A, int ctas)
        : per((A.groups + 31) >> 5), longest(0), before(0), mine(0), total(0) {
        const int lane = threadIdx.x & 31;
        // This lane's first group, which is all it has up to 32: nothing is read twice.
        const PrefixGroup first(A, lane * per);
        auto each = [&](auto f) {
            f(first);
            for (int k = 1; k < per; ++k) f(PrefixGroup(A, lane * per + k));
        };
        // In 32 bits: a lane's sums end at kMany, far more than there may be chunks.
        constexpr int kMany = 1 << 25;
        auto items = [&](const PrefixGroup& gr) { return gr.nb ? min(gr.pairs * A.Hkv, 4096) : 0; };   // of 8192 blocks at most: 2^25
        int own = 0;
        each([&](const PrefixGroup& gr) { own = min(own + items(gr) * gr.nb, kMany); });
        const unsigned blocks = __reduce_add_sync(0xffffffffu, (unsigned)own);
        auto fits = [&](int length) {   // chunks of that length, a CTA each
            int n = 0;
            each([&](const PrefixGroup& gr) { n = min(n + items(gr) * chunks(gr, length), kMany); });
            return __reduce_add_sync(0xffffffffu, (unsigned)n) <= (unsigned)ctas;
        };
        const int mean = (int)(blocks / (unsigned)ctas);
        if (blocks && fits(mean + mean / 4 + 1)) {
            int lo = mean > 0 ? mean : 1, hi = mean + mean / 4 + 1;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (fits(mid)) hi = mid; else lo = mid + 1;
            }
            longest = lo;
        }
        each([&](const PrefixGroup& gr) { mine += part(A, gr); });
        long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += y;
        }
        before = upto - mine;
        total = __shfl_sync(0xffffffffu, upto, 31);
    }
    // The group of chunk or place `at` < total, which becomes that within the group.  (It ends whatever the lengths say: they
    // may be written meanwhile by a program that does not wait for the call.)
    __device__ __forceinline__ int group_at(const PrefixGeom& A, long long& at) const {
        const int l = __ffs(__ballot_sync(0xffffffffu, at < before + mine)) - 1;
        at -= __shfl_sync(0xffffffffu, before, l);
        int r = l * per;
        for (; r < A.groups; ++r) {
            const long long here = part(A, PrefixGroup(A, r));
            if (at < here) break;
            at -= here;
        }
        return r;
    }
    // Chunks or places of the groups before r, by a whole warp.
    __device__ __forceinline__ long long parts_before(const PrefixGeom& A, int r) const {
        const int l = r / per;
        return __shfl_sync(0xffffffffu, before, l) +
               sum_by_lanes(l * per, r, [&](int k) { return part(A, PrefixGroup(A, k)); });
    }
};
__device__ __forceinline__ long long group_share(long long total, int cta, int ctas) { return total * cta / ctas; }

// Where the sums of sequence s are.
__device__ __forceinline__ PrefixPlan plan_of(const PrefixGeom& A, const GroupList& list, int s) {
    PrefixPlan p{};
    int lo = 0, hi = A.groups;   // the last group that begins at or before s
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (__ldg(&A.cu[mid]) <= s) lo = mid; else hi = mid - 1;
    }
    const PrefixGroup gr(A, lo);
    if (gr.places() == 0 || s < gr.q0 || s >= gr.q0 + gr.n) return p;   // behind the last group there is none
    const int seat = s - gr.q0, pair = seat / (2 * A.nq);
    const long long before = list.parts_before(A, lo);
    p.base = (seat - pair * 2 * A.nq) * A.g;
    if (list.longest) {
        p.n = GroupList::chunks(gr, list.longest);
        p.step = gr.pairs;
        p.at = before + pair;
        p.at_step = (long long)p.n * gr.pairs;
    } else {
        p.n = gr.nb;
        p.total = list.total;
        p.at = before + (long long)pair * gr.places() + PrefixGroup::kCost;
        p.at_step = (long long)gr.pairs * gr.places();
        p.base += gr.first_row(A, 0, pair);
        p.base_step = gr.n * A.g;
    }
    return p;
}

// The sums of the first query row of (sequence, KV head): n of them, each in a row of its own.
struct PrefixParts {
    int n, c0, step, base, ctas;   // of CTAs c0, c0 + step, ..
    long long total;
    __device__ __forceinline__ PrefixParts(const PrefixPlan& p, int h, int num_ctas)
        : n(p.n), c0(0), step(1), base(p.base + h * p.base_step), ctas(num_ctas), total(p.total) {
        const long long at = p.at + h * p.at_step;
        if (total == 0) {
            c0 = (int)at;
            step = p.step;
        } else {
            c0 = (int)(((at + 1) * ctas - 1) / total);
            n = (int)(((at + p.n) * ctas - 1) / total) - c0 + 1;
        }
    }
    // Row of the k-th; -1: the CTA's share is empty, as there are more CTAs than blocks.
    __device__ __forceinline__ int row(int k) const {
        const int cta = c0 + k * step;
        return total == 0 || group_share(total, cta, ctas) < group_share(total, cta + 1, ctas) ? base + 2 * kPrefixTile * cta : -1;
    }
};

}  // namespace kvec
