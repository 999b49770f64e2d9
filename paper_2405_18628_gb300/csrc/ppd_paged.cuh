// ppd_paged.cuh -- a cache in pages, for the attention kernels: what a launch over pages
// has in addition, and the copies of a tile of 128 keys out of the pages that hold it.
//
// A pool is [L][n_pages][H][page][D]; sequence b's row r is row r mod page of page
// table[b][r / page] in every layer.  The pool's tensor map has a (layer, page, head) as its
// depth, so a tile is 128 / page boxes of page rows at depths that the table gives (one box where
// a page holds 128 rows or more).  Boxes start on multiples of eight rows of 128 bytes, so that
// the swizzled tile is the one that a contiguous cache gives.  A lane of a producer's warp
// looks up a box's page: 8-row pages take 16 of them.
//
// A table entry that names no page reads as zeros (a coordinate past the tensor's end), and the
// sequence's status says so; nothing is read outside the pool.
#pragma once

#include "ppd_device.cuh"
#include "ppd_kernels.h"

#include <type_traits>

namespace ppd {

template <bool PAGED>
using AttnParamsOf = std::conditional_t<PAGED, PagedParams, AttnParams>;
template <bool PAGED>
using OutOf = std::conditional_t<PAGED, __nv_bfloat16, float>;

// Query rows of a slice.
template <bool PAGED>
PPD_DEV int query_rows(const AttnParamsOf<PAGED> &p)
{
    if constexpr (PAGED) return p.rows;
    else return p.T;
}

// A slice's row of the table, and the depth of its layer's and head's page 0.
struct PageUnit {
    const int32_t *row;
    int depth0;
    PPD_DEV PageUnit(const PagedParams &p, int lbh, int b)
    {
        const int l = lbh / (p.H * p.B), h = lbh % p.H;
        row = p.table + (size_t)b * p.max_pages;
        depth0 = l * p.n_pages * p.H + h;   // the host has checked that depths fit 32 bits
    }
};

PPD_DEV int page_depth(const PagedParams &p, const PageUnit &u, int id)
{
    return (unsigned)id < (unsigned)p.n_pages ? u.depth0 + id * p.H : p.n_depth;
}

// This lane's box of the tile that starts at key `row` of P: the depth of its page, or -1 where
// the lane has no box (or none with a key below P).
PPD_DEV int page_coord(const PagedParams &p, const PageUnit &u, int row, int P, int lane)
{
    const int r = row + (lane << p.box_shift);
    if (r >= P || r >= row + 128) return -1;
    return page_depth(p, u, ld_input(u.row + (r >> p.page_shift)));
}

// The tile itself, by a converged warp: every box that holds a key below P (`more`: bytes that the
// caller copies besides).  One elected lane issues the copies of all of them, from warp-uniform code: lanes
// that each copied a box took 115 cycles a box, one after the other (with one producer, 48 requests of up to
// 8192 rows in pages of 16: 224 -> 180 us).
template <int DCH>
PPD_DEV void load_page_tile(const PagedParams &p, const CUtensorMap *map, uint8_t *dst, uint32_t group_bytes, uint64_t *full,
                            int depth, int row, int P, uint64_t policy, uint32_t more = 0)
{
    const int n = warp_uniform((max(0, min(128, P - row)) + (1 << p.box_shift) - 1) >> p.box_shift);
    const uint32_t box_bytes = 128u << p.box_shift;
    const int y = warp_uniform(row & ((1 << p.page_shift) - 1));
    if (elect_one()) mbar_arrive_expect_tx(full, (uint32_t)n * DCH * box_bytes + more);
    __syncwarp();
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const int z = __shfl_sync(0xffffffffu, depth, i);
        if (elect_one()) {
#pragma unroll
            for (int c = 0; c < DCH; ++c) tma_load_3d(dst + c * group_bytes + i * box_bytes, map, full, c * 64, y, z, policy);
        }
    }
    __syncwarp();
}

// Before the wait of a chained launch (one warp): ask L2 for the prefix tiles [j, j + n) of unit
// u, K and V, by lengths and tables that may still be changing.  Only a
// hint, as prefetch_first_tiles.
template <int DCH>
PPD_DEV void prefetch_pages(const PagedParams &p, int lane, const CUtensorMap *kc, const CUtensorMap *vc, int u, int j, int n)
{
    if (u >= p.n_units) return;
    const int lbh = u / p.n_qb, b = (lbh / p.H) % p.B;
    const int P = min(max(ld_relaxed_gpu_s32(p.prefix_len + b), 0), p.S_max);
    const PageUnit pu(p, lbh, b);
    for (int row = j * 128; row < min(P, (j + n) * 128); row += 128) {
        const int r = row + (lane << p.box_shift);
        if (r >= P || r >= row + 128) continue;
        const int depth = page_depth(p, pu, ld_relaxed_gpu_s32(pu.row + (r >> p.page_shift)));
        if (depth == p.n_depth) continue;
        for (int c = 0; c < DCH; ++c) {
            tma_prefetch_l2_3d(kc, c * 64, r & ((1 << p.page_shift) - 1), depth);
            tma_prefetch_l2_3d(vc, c * 64, r & ((1 << p.page_shift) - 1), depth);
        }
    }
}

// The statuses, by one warp a CTA, sequence b by CTA b mod grid: none yet, before its copies; after them a
// malformed tree, then a prefix outside the table, or an entry of it that names no page.  (By a maximum: the
// status of a wait that ran out meanwhile, in any CTA, is the largest, and stays.)
PPD_DEV void paged_status_none(const PagedParams &p, int lane)
{
    for (int b = blockIdx.x + lane * gridDim.x; b < p.B; b += 32 * gridDim.x) p.dev_status[b] = kOk;
    __syncwarp();
}

PPD_DEV void paged_status_warp(const PagedParams &p, int lane)
{
    for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
        bool bad = false, gap = false;
        for (int i = lane; i < p.T; i += 32) {
            const int pa = ld_input(p.parent + (size_t)b * p.T + i);
            bad |= i == 0 ? pa != -1 : (pa < 0 || pa >= i);
        }
        const int P = ld_input(p.prefix_len + b);
        const bool out = P < 0 || P > p.S_max;
        if (!out) {
            const int32_t *row = p.table + (size_t)b * p.max_pages;
            const int n = (P + (1 << p.page_shift) - 1) >> p.page_shift;
#pragma unroll 4
            for (int i = lane; i < n; i += 32) gap |= (unsigned)ld_input(row + i) >= (unsigned)p.n_pages;
        }
        bad = __any_sync(0xffffffffu, bad);
        gap = __any_sync(0xffffffffu, gap);
        if (lane == 0 && (bad || out || gap)) atomicMax(p.dev_status + b, (int)(bad ? kErrTree : kErrCapacity));
    }
}

}  // namespace ppd
