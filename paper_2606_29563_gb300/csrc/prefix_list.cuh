// The work on prefixes that groups of sequences share: the list of the 128-key blocks of all (group, KV head, pair of
// 128-row tiles) items, of which every CTA of prefill_kernel's PAGED form takes an even share, and where it leaves the
// sums that shared_join_kernel reads.
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

// The list as a warp sees it: lane l holds the groups l * per .. l * per + per - 1, over all heads and pairs.
struct GroupList {
    int per;
    long long before, mine, total;   // places: of the lanes before, of this lane, of all
    __device__ __forceinline__ GroupList(const PrefixGeom& A) : per((A.groups + 31) >> 5), before(0), mine(0), total(0) {
        const int lane = threadIdx.x & 31;
        for (int k = 0; k < per; ++k) {
            const PrefixGroup gr(A, lane * per + k);
            mine += (long long)gr.places() * gr.pairs * A.Hkv;
        }
        long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += y;
        }
        before = upto - mine;
        total = __shfl_sync(0xffffffffu, upto, 31);
    }
    // The group of place `at` < total, which becomes the place within the group.
    __device__ __forceinline__ int group_at(const PrefixGeom& A, long long& at) const {
        const int l = __ffs(__ballot_sync(0xffffffffu, at < before + mine)) - 1;
        at -= __shfl_sync(0xffffffffu, before, l);
        for (int r = l * per;; ++r) {
            const PrefixGroup gr(A, r);
            const long long here = (long long)gr.places() * gr.pairs * A.Hkv;
            if (at < here) return r;
            at -= here;
        }
    }
    __device__ __forceinline__ long long places_before(const PrefixGeom& A, int r) const {
        const int l = r / per;
        long long b = __shfl_sync(0xffffffffu, before, l);
        for (int k = l * per; k < r; ++k) {
            const PrefixGroup gr(A, k);
            b += (long long)gr.places() * gr.pairs * A.Hkv;
        }
        return b;
    }
};
__device__ __forceinline__ long long group_share(long long total, int cta, int ctas) { return total * cta / ctas; }

// The sums of query row (s, hq): those of CTAs c0 .. c1, base + 2 kPrefixTile c the row of CTA c's.
struct PrefixParts {
    int c0 = 0, c1 = -1, base = 0;
    long long total;
    __device__ __forceinline__ PrefixParts(const PrefixGeom& A, int s, int h, int ctas) {
        const GroupList list(A);
        total = list.total;
        int lo = 0, hi = A.groups;   // the last group that begins at or before s
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (__ldg(&A.cu[mid]) <= s) lo = mid; else hi = mid - 1;
        }
        const PrefixGroup gr(A, lo);
        if (gr.places() == 0 || s < gr.q0 || s >= gr.q0 + gr.n) return;   // behind the last group there is none
        const int seat = s - gr.q0, pair = seat / (2 * A.nq);
        const long long at = list.places_before(A, lo) + (long long)(h * gr.pairs + pair) * gr.places() + PrefixGroup::kCost;
        c0 = (int)(((at + 1) * ctas - 1) / total);
        c1 = (int)(((at + gr.nb) * ctas - 1) / total);
        base = gr.first_row(A, h, pair) + (seat - pair * 2 * A.nq) * A.g;
    }
    // -1: the CTA's share is empty, as there are more CTAs than blocks.
    __device__ __forceinline__ int row(int cta, int ctas) const {
        return group_share(total, cta, ctas) < group_share(total, cta + 1, ctas) ? base + 2 * kPrefixTile * cta : -1;
    }
};

}  // namespace kvec
