// ppd_kv4_wide.cu -- the tree's attention over a 4-bit cache on the 5th-generation tensor cores,
// for more query rows than the few-row kernel (ppd_kv4.cu) takes.
//
// One persistent CTA per SM walks an equal share of all key tiles (the work split of
// ppd_attention_common.cuh: a unit is a slice's block of up to 64 query rows, a row being
// one of the G query heads' tree tokens; tiles of 128 keys, the tree's last).  Per tile:
//
//   K     four warps make a tile's values from its codes, a key row a thread, and store
//         them into tensor memory: the A operand of S^T = K Q^T needs no shared memory
//   V     the same rows into shared memory, the A operand of O^T += V^T [P_hi | P_lo]^T
//   P     by eight softmax warps as in the bf16 key-row kernel (ppd_attention.cu): a key row a
//         thread, lazy maxima, probabilities in two bf16 terms
//
// The converting warps fetch their own rows by asynchronous copies, two tiles ahead, so the
// codes pass shared memory once and meet no barrier on their way in.
//
// Bound by the softmax warps, which the scores never wait for: some 1100 of a tile's 1760 cycles (64
// query rows, D = 128) are the probabilities' instructions, the rest their way from and to the
// tensor cores and the tile's vote; shared memory's loads and stores take some 800 cycles beside
// the products' own reads, the products a third.  A unit's first scores, its tree, row sums and output
// cost four tiles more: 1024 slices of 2048 keys 140 us, 2.5 TB/s, 0.49 PFLOP/s; eight sequences of
// up to 16,384 keys (4 x 32 slices each) 604 us, 2.5 TB/s, 0.57 PFLOP/s.
#include "ppd_attention_common.cuh"
#include "ppd_kv4.cuh"

#include <cmath>

namespace ppd {

template <int D_, int TP_>
struct Kv4Wide {
    static constexpr int D = D_, TP = TP_;        // TP: query columns (32 or 64)
    static constexpr int KT = 128;                // keys per tile
    static constexpr int DCH = D / 64;
    static constexpr int NWG = 2, NC = TP / NWG;  // softmax warpgroups, columns of each
    // softmax warps, four warps converting K, four converting V, then three that bring Q and the issuer
    static constexpr int SW = 8, KW = SW, VW = KW + 4, QW = VW + 4, NQ = 3, IW = QW + NQ;
    static constexpr int THREADS = (IW + 1) * 32;
    // registers a thread: 20 warps start with 96 and share the same total out anew (144 to 176 for the
    // softmax: 140 to 148 us and 604 to 652 for those below, the compiler's order of the loop more
    // than the registers)
    static constexpr int SOFTMAX_REGS = 168, CONVERT_REGS = 56, OTHER_REGS = 32;
    static_assert(2 * SOFTMAX_REGS + 2 * CONVERT_REGS + OTHER_REGS <= 5 * 96, "register shares");
    static constexpr int STAGES = 3;              // tiles of codes in a converting warp's ring
    static constexpr int QS = 2, PS = 2, VS = 2, OB = 2;
    static constexpr uint32_t GROUP_BYTES = KT * 128;
    static constexpr uint32_t TILE_BYTES = KT * D * 2;
    static constexpr uint32_t Q_GROUP_BYTES = TP * 128;
    static constexpr uint32_t Q_BYTES = TP * D * 2;
    static constexpr uint32_t P_BYTES = (2 * TP / 64) * GROUP_BYTES;
    static constexpr int RB = D / 2, SB = D / kKv4Group;
    static constexpr uint32_t CODES = 32 * RB;    // a warp's rows of a tile
    static constexpr uint32_t STAGE = CODES + 128;

    static constexpr uint32_t OFF_Q = 0;
    static constexpr uint32_t OFF_P = OFF_Q + QS * Q_BYTES;
    static constexpr uint32_t OFF_V = OFF_P + PS * P_BYTES;
    static constexpr uint32_t OFF_RING = OFF_V + VS * TILE_BYTES;
    static constexpr uint32_t OFF_BAR = OFF_RING + 8 * STAGES * STAGE;
    static constexpr int B_QFULL = 0, B_QEMPTY = B_QFULL + QS, B_KFULL = B_QEMPTY + QS, B_VFULL = B_KFULL + 2,
                         B_SFULL = B_VFULL + VS, B_PFULL = B_SFULL + 2, B_PFREE = B_PFULL + 2, B_DRAIN = B_PFREE + 2,
                         NBAR = B_DRAIN + 1;
    static constexpr uint32_t OFF_TMEMPTR = OFF_BAR + NBAR * 8;
    static constexpr uint32_t OFF_ABORT = OFF_TMEMPTR + 4;
    static constexpr uint32_t OFF_NM = (OFF_ABORT + 4 + 15) & ~15u;   // [TP] minus the running references
    static constexpr uint32_t OFF_L = OFF_NM + TP * 4;                // [OB][TP] row sums (1 / sum of a whole unit)
    static constexpr uint32_t OFF_MX = OFF_L + OB * TP * 4;           // [OB][TP] references of a part
    static constexpr uint32_t OFF_RED = OFF_MX + OB * TP * 4;         // [NWG][4][NC]
    static constexpr uint32_t OFF_RANGE = (OFF_RED + NWG * 4 * NC * 4 + 15) & ~15u;
    static constexpr uint32_t OFF_PARENT = (OFF_RANGE + sizeof(WorkRange) + 15) & ~15u;   // [NWG][kMaxTree]
    static constexpr uint32_t SMEM_BYTES = OFF_PARENT + NWG * kMaxTree * 4;
    // tensor memory: K0 | K1 | S0 | S1 | O0 (hi | lo) | O1
    static constexpr uint32_t T_K = 0, T_S = D, T_O = T_S + 2 * TP, TMEM_COLS = 512;

    static_assert(SMEM_BYTES <= 232448, "shared memory budget");
    static_assert((OFF_P | OFF_V) % 1024 == 0 && OFF_RING % 16 == 0, "aligned operand tiles");
    static_assert(T_O + OB * 2 * TP <= TMEM_COLS, "tensor memory budget");
};

// This CTA's units one by one, as SegIter hands them out: whole ones round-robin, or (SPLIT) those
// of its range of tiles.  The sequence of a unit comes by adding where SegIter divides: every
// role does this between two units, and short contexts feel it (2000 cycles a unit).
template <bool SPLIT>
struct UnitIter {
    int u, j0, left;
    int r, b;                         // u = x d + r, d units a (layer, sequence); b = x % B
    int d, step_r, step_b;
    PPD_DEV UnitIter(const AttnParams &p, const WorkRange &w)
    {
        u = SPLIT ? w.u_first : (int)blockIdx.x;
        j0 = SPLIT ? w.j_first : 0;
        left = SPLIT ? w.n_tiles : 0;
        const int step = SPLIT ? 1 : (int)gridDim.x;
        d = p.H * p.n_qb;
        r = u % d;
        b = u / d % p.B;
        step_r = step % d;
        step_b = step / d % p.B;
    }
    PPD_DEV bool next(const AttnParams &p, Seg &s)
    {
        if ((SPLIT && left <= 0) || u >= p.n_units) return false;
        s.u = u;
        s.ui.lbh = p.n_qb == 1 ? u : u / p.n_qb;
        s.ui.qb = u - s.ui.lbh * p.n_qb;
        s.ui.b = b;
        s.ui.P_raw = ld_input(p.prefix_len + b);
        s.ui.P = min(max(s.ui.P_raw, 0), p.S_max);
        s.ui.n_pref = (s.ui.P + 127) >> 7;
        s.ui.n_tiles = s.ui.n_pref + p.n_tt;
        s.j0 = j0;
        s.j1 = SPLIT ? min(s.ui.n_tiles, j0 + left) : s.ui.n_tiles;
        if (s.j1 <= s.j0) {   // cannot happen with a consistent plan; never loop on it
            left = 0;
            u = p.n_units;
            return false;
        }
        left -= s.j1 - s.j0;
        j0 = 0;
        u += SPLIT ? 1 : (int)gridDim.x;
        r += step_r;
        b += step_b;
        if (r >= d) r -= d, ++b;
        if (b >= p.B) b -= p.B;
        return true;
    }
};

// The tiles of a CTA's range one by one.
template <bool SPLIT>
struct TileWalk {
    UnitIter<SPLIT> it;
    Seg sg;
    int j = 0, end = 0;
    PPD_DEV TileWalk(const AttnParams &p, const WorkRange &w) : it(p, w) {}
    PPD_DEV bool next(const AttnParams &p)   // sg and j then name a tile
    {
        if (++j >= end) {
            if (!it.next(p, sg)) return false;
            j = sg.j0;
            end = sg.j1;
        }
        return true;
    }
};

template <int D, int TP, bool SPLIT>
__global__ void __launch_bounds__(Kv4Wide<D, TP>::THREADS, 1)
kv4_attention_wide_kernel(const AttnParams p, const Kv4AttnParams x)
{
    using Lay = Kv4Wide<D, TP>;
    using VPos = RingPos<Lay::VS>;
    constexpr int NC = Lay::NC;
    using Cols = uint32_t[Lay::NC];
    using Probs = uint64_t[Lay::NC / 2];
    extern __shared__ __align__(1024) uint8_t smem[];
    if (smem_addr(smem) & 1023u) {   // the swizzled tiles' alignment: uniform over the CTA
        if (threadIdx.x == 0)
            for (int b = 0; b < p.B; ++b) p.dev_status[b] = kErrUnsupported;
        return;
    }
    uint64_t *bars = reinterpret_cast<uint64_t *>(smem + Lay::OFF_BAR);
    uint32_t *tmem_ptr = reinterpret_cast<uint32_t *>(smem + Lay::OFF_TMEMPTR);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + Lay::OFF_ABORT);
    const int warp = warp_uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int T = p.T, R = x.G * x.T;

    if (threadIdx.x == 0) {
        for (int i = 0; i < Lay::NBAR; ++i) {
            uint32_t count = i < Lay::B_QEMPTY ? Lay::NQ : 1;
            if (i >= Lay::B_KFULL && i < Lay::B_SFULL) count = 4;   // K and V tiles
            if (i >= Lay::B_PFULL && i < Lay::B_PFULL + 2) count = Lay::SW;
            mbar_init(bars + i, count);
        }
        *abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == Lay::IW) {
        tmem_alloc(tmem_ptr, Lay::TMEM_COLS);
        tmem_relinquish();
    }
    pdl_wait();
    WorkRange *wr_s = reinterpret_cast<WorkRange *>(smem + Lay::OFF_RANGE);
    if (warp == Lay::QW) {
        const WorkRange w = plan_range(p, lane);
        if (lane == 0) {
            *wr_s = w;
            if (SPLIT) p.split_rec[blockIdx.x].u = -1;
        }
    }
    pdl_release();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_ptr;
    const WorkRange &wr = *wr_s;

    if (warp >= Lay::KW && warp < Lay::QW) {
        // ------------------------------------------------------------ converting warps
        reg_dec<Lay::CONVERT_REGS>();
        const bool kv = warp >= Lay::VW;         // V, or K
        const int wq = warp & 3;                 // this warp's rows of a tile, and lanes of tensor memory
        const int t = wq * 32 + lane;
        const uint8_t *codes = kv ? x.v_cache : x.k_cache, *scales = kv ? x.v_scale : x.k_scale;
        const void *tree_rows = kv ? x.v_tree : x.k_tree;
        const uint32_t ring = smem_addr(smem) + Lay::OFF_RING + (uint32_t)(warp - Lay::KW) * Lay::STAGES * Lay::STAGE;
        const uint32_t k_mem = tmem_base + ((uint32_t)(wq * 32) << 16) + Lay::T_K;
        const uint32_t v_row = smem_addr(smem) + Lay::OFF_V + (uint32_t)(t >> 3) * 1024u + (uint32_t)(t & 7) * 128u;
        constexpr int UPR = Lay::RB / 16;        // 16-byte pieces of a row's codes, 32 channels each
        TileWalk<SPLIT> ahead(p, wr), at(p, wr);
        bool more = true;
        // piece i of this lane: row i * 32 / UPR + lane / UPR of the warp's 32, 512 bytes on from
        // piece i - 1 on both sides.  A thread reads one row: eight rows' equal pieces lie in
        // different banks.
        const int f_row = lane / UPR;
        const uint32_t f_to = (uint32_t)(f_row * UPR + ((lane % UPR) ^ (UPR == 4 ? (f_row >> 1) & 3 : (f_row >> 2) & 1))) * 16;
        auto fetch = [&](int stage) {
            if (more) more = ahead.next(p);
            if (more) {
                const UnitInfo &ui = ahead.sg.ui;
                const uint32_t dst = ring + stage * Lay::STAGE;
                if (ahead.j < ui.n_pref) {
                    const int k0 = ahead.j * Lay::KT + wq * 32, n = ui.P - k0;   // rows from k0 on
                    const size_t row0 = (size_t)ui.lbh * p.S_max + (n > 0 ? k0 : 0);
                    const uint8_t *src = codes + row0 * Lay::RB + lane * 16, *sc = scales + row0 * Lay::SB;
                    if (D == 128 && n >= 32) {
#pragma unroll
                        for (int i = 0; i < UPR; ++i) cp_async16(dst + f_to + i * 512, src + i * 512, 16u);
                        cp_async4(dst + Lay::CODES + lane * 4, sc + lane * 4, 4u);
                    } else {
#pragma unroll
                        for (int i = 0; i < UPR; ++i) {
                            const bool in = i * 32 / UPR + f_row < n;
                            cp_async16(dst + f_to + i * 512, in ? src + i * 512 : codes, in ? 16u : 0u);
                        }
                        const bool in = lane < n;
                        const size_t a = (row0 * Lay::SB + (in ? lane * Lay::SB : 0)) & ~(size_t)3;
                        const size_t left = x.scale_bytes - a;
                        cp_async4(dst + Lay::CODES + lane * 4, scales + a, in ? (left < 4 ? (uint32_t)left : 4u) : 0u);
                    }
                } else {
                    // a tree tile is read from L2 when its turn comes
                    const int jt = (ahead.j - ui.n_pref) * Lay::KT + t;
                    const int bytes = x.f32 ? 4 * D : 2 * D;
                    const uint8_t *row = reinterpret_cast<const uint8_t *>(tree_rows) + ((size_t)ui.lbh * T + (jt < T ? jt : 0)) * bytes;
                    if (jt < T)
                        for (int i = 0; i < bytes; i += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + i));
                }
            }
            cp_async_commit();
        };
#pragma unroll
        for (int s = 0; s < Lay::STAGES - 1; ++s) fetch(s);
        int stage = 0;
        for (int g = 0; at.next(p); ++g) {
            fetch((stage + Lay::STAGES - 1) % Lay::STAGES);
            const int buf = g & 1;
            const bool tree = at.j >= at.sg.ui.n_pref;
            auto store = [&](int c, const uint32_t (&r)[16]) {   // channels 32 c ..
                if (!kv) {
                    tmem_st16(k_mem + (uint32_t)buf * (D / 2) + c * 16, r);
                } else {
                    const uint32_t row = v_row + buf * Lay::TILE_BYTES + (c >> 1) * Lay::GROUP_BYTES;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        st_shared_v4(row + (uint32_t)(((4 * (c & 1) + i) ^ (t & 7)) << 4), r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
                }
            };
            // the buffer is free once tile g - 2's scores (K), or its product with P (V), are done
            uint64_t *free_bar = bars + (kv ? Lay::B_PFREE : Lay::B_SFULL) + buf;
            if (!tree) {
                cp_async_wait<Lay::STAGES - 1>();
                __syncwarp();
                const uint32_t src = ring + stage * Lay::STAGE;
                // (D = 64: a word of scales holds an even and an odd row's)
                const uint32_t odd = D == 64 ? (uint32_t)(((size_t)at.sg.ui.lbh * p.S_max + (size_t)at.j * Lay::KT + t) & 1) * 16u : 0u;
                const uint32_t sc = ld_shared_u32(src + Lay::CODES + lane * 4) >> odd;
                if (g >= 2) mbar_wait(free_bar, ((g >> 1) - 1) & 1, abort_flag);
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < UPR; ++c) {
                    const uint4 w = ld_shared_u128(src + (uint32_t)(lane * UPR + (UPR == 4 ? c ^ ((lane >> 1) & 3) : c ^ ((lane >> 2) & 1))) * 16);
                    const Kv4Scale k = kv4_scales(((sc >> (8 * c)) & 0xFFu) * 0x10001u);
                    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
                    uint32_t r[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        uint32_t v[4];
                        kv4_word(u[i >> 2], k, v);
                        r[i] = v[0], r[i + 1] = v[1], r[i + 2] = v[2], r[i + 3] = v[3];
                    }
                    store(c, r);
                }
            } else {
                const int jt = (at.j - at.sg.ui.n_pref) * Lay::KT + t;   // tree key
                const bool in = jt < T;
                const size_t row = ((size_t)at.sg.ui.lbh * T + (in ? jt : 0)) * D;
                if (g >= 2) mbar_wait(free_bar, ((g >> 1) - 1) & 1, abort_flag);
                tc_fence_after();
                if (!x.f32) {
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t r[16];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint4 v = in ? ld_input(reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(tree_rows) + row + 32 * c) + i)
                                               : make_uint4(0, 0, 0, 0);
                            r[4 * i] = v.x, r[4 * i + 1] = v.y, r[4 * i + 2] = v.z, r[4 * i + 3] = v.w;
                        }
                        store(c, r);
                    }
                } else {
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        const float4 *src = reinterpret_cast<const float4 *>(tree_rows) + (row >> 2) + 8 * c;
                        uint32_t r[16];
#pragma unroll
                        for (int h = 0; h < 8; h += 4) {
                            float4 v[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) v[i] = in ? ld_input(src + h + i) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                            for (int i = 0; i < 4; ++i) r[2 * (h + i)] = bf16x2(v[i].x, v[i].y), r[2 * (h + i) + 1] = bf16x2(v[i].z, v[i].w);
                        }
                        store(c, r);
                    }
                }
            }
            if (!kv) {
                tmem_wait_st();
                tc_fence_before();
            } else {
                fence_proxy_async_smem();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + (kv ? Lay::B_VFULL : Lay::B_KFULL) + buf);
            stage = (stage + 1) % Lay::STAGES;
        }
        cp_async_wait<0>();
    } else if (warp < Lay::IW && warp >= Lay::QW) {
        // ------------------------------------------------------------ Q warps, statuses
        reg_dec<Lay::OTHER_REGS>();
        if (warp == Lay::QW) status_warp(p, lane);
        const int i0 = (warp - Lay::QW) * 32 + lane;
        int k = 0;
        UnitIter<SPLIT> it(p, wr);
        for (Seg sg; it.next(p, sg); ++k) {
            const int qs = k & 1;
            mbar_wait(bars + Lay::B_QEMPTY + qs, ((k >> 1) & 1) ^ 1, abort_flag);
            const uint32_t dst = smem_addr(smem) + Lay::OFF_Q + qs * Lay::Q_BYTES;
            const int r0 = sg.ui.qb * TP;
            const size_t row0 = (size_t)sg.ui.lbh * R + r0;
            constexpr int CPR = D / 8;   // 16-byte chunks of a row
            auto chunk_at = [&](int row, int c) {
                return dst + (uint32_t)(c >> 3) * Lay::Q_GROUP_BYTES + (uint32_t)(row >> 3) * 1024u + (uint32_t)(row & 7) * 128u +
                       (uint32_t)(((c & 7) ^ (row & 7)) << 4);
            };
            if (!x.f32) {   // every chunk on its way at once
                const uint8_t *src = reinterpret_cast<const uint8_t *>(x.q) + row0 * D * 2;
#pragma unroll 4
                for (int i = i0; i < TP * CPR; i += Lay::NQ * 32) {
                    const bool in = r0 + i / CPR < R;
                    cp_async16(chunk_at(i / CPR, i % CPR), in ? src + (size_t)i * 16 : reinterpret_cast<const uint8_t *>(x.q), in ? 16u : 0u);
                }
                cp_async_commit();
                cp_async_wait<0>();
            } else {   // two chunks' loads in flight
                const float4 *src = reinterpret_cast<const float4 *>(x.q) + row0 * (D / 4);
#pragma unroll 1
                for (int i = i0; i < TP * CPR; i += 2 * Lay::NQ * 32) {
                    float4 v[4];
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const int c = i + (h >> 1) * Lay::NQ * 32;
                        v[h] = c < TP * CPR && r0 + c / CPR < R ? ld_input(src + 2 * c + (h & 1)) : make_float4(0.f, 0.f, 0.f, 0.f);
                    }
#pragma unroll
                    for (int h = 0; h < 4; h += 2) {
                        const int c = i + (h >> 1) * Lay::NQ * 32;
                        if (c < TP * CPR)
                            st_shared_v4(chunk_at(c / CPR, c % CPR), bf16x2(v[h].x, v[h].y), bf16x2(v[h].z, v[h].w),
                                         bf16x2(v[h + 1].x, v[h + 1].y), bf16x2(v[h + 1].z, v[h + 1].w));
                    }
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + Lay::B_QFULL + qs);
        }
    } else if (warp == Lay::IW) {
        // ------------------------------------------------------------ MMA issuer
        reg_dec<Lay::OTHER_REGS>();
        constexpr uint32_t idesc_qk = make_idesc_bf16(128, TP, 0, 0);
        constexpr uint32_t idesc_pv = make_idesc_bf16(128, 2 * TP, 1, 1);
        const uint32_t tmem = warp_uniform(tmem_base);
        const uint32_t s0 = warp_uniform(smem_addr(smem));
        constexpr uint32_t v_lbo = (D == 128) ? Lay::GROUP_BYTES : 0u;   // D = 64: both M halves read the same rows
        const uint64_t dq0 = make_smem_desc(s0 + Lay::OFF_Q, 16, 1024);
        const uint64_t dv0 = make_smem_desc(s0 + Lay::OFF_V, v_lbo, 1024);
        const uint64_t dp0 = make_smem_desc(s0 + Lay::OFF_P, Lay::GROUP_BYTES, 1024);
        VPos vp;
        int gp = 0;
        auto issue_pv = [&](bool first, uint32_t t_o) {
            const int ps = gp & 1;
            mbar_wait(bars + Lay::B_VFULL + vp.slot, vp.phase, abort_flag);
            mbar_wait(bars + Lay::B_PFULL + ps, (gp >> 1) & 1, abort_flag);
            tc_fence_after();
            const bool dead = warp_uniform(*abort_flag) != 0;
            if (elect_one()) {
                if (!dead) {
                    const uint64_t a0 = desc_advance(dv0, vp.slot * Lay::TILE_BYTES);
                    const uint64_t b0 = desc_advance(dp0, ps * Lay::P_BYTES);
#pragma unroll
                    for (int kk = 0; kk < Lay::KT / 16; ++kk)
                        umma_bf16(t_o, desc_advance(a0, kk * 2048), desc_advance(b0, kk * 2048), idesc_pv,
                                  (first && kk == 0) ? 0u : 1u);
                }
                umma_commit(bars + Lay::B_PFREE + ps);   // P's tile and V's slot (the same parity) are free
            }
            __syncwarp();
            vp.advance();
            ++gp;
        };
        int g = 0, k = 0;
        bool prev_first = false;
        uint32_t prev_to = 0;
        UnitIter<SPLIT> it(p, wr);
        for (Seg sg;; ++k) {
            const int n = warp_uniform(it.next(p, sg) ? sg.j1 - sg.j0 : 0);
            if (n == 0) break;
            const int qs = k & 1;
            const uint32_t t_o = tmem + Lay::T_O + (uint32_t)(k & 1) * 2 * TP;
            mbar_wait(bars + Lay::B_QFULL + qs, (k >> 1) & 1, abort_flag);
            for (int j = 0; j < n; ++j, ++g) {
                const int sb = g & 1;
                mbar_wait(bars + Lay::B_KFULL + sb, (g >> 1) & 1, abort_flag);
                tc_fence_after();
                const bool dead = warp_uniform(*abort_flag) != 0;
                if (elect_one()) {
                    if (!dead) {
                        const uint32_t a0 = tmem + Lay::T_K + sb * (D / 2);
                        const uint64_t b0 = desc_advance(dq0, qs * Lay::Q_BYTES);
                        const uint32_t d_s = tmem + Lay::T_S + sb * TP;
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk)
                            umma_bf16_ta(d_s, a0 + kk * 8, desc_advance(b0, (kk >> 2) * Lay::Q_GROUP_BYTES + (kk & 3) * 32), idesc_qk,
                                         kk > 0 ? 1u : 0u);
                    }
                    umma_commit(bars + Lay::B_SFULL + sb);
                    if (j == n - 1) umma_commit(bars + Lay::B_QEMPTY + qs);
                }
                __syncwarp();
                if (g > 0) issue_pv(prev_first, prev_to);
                prev_first = (j == 0);
                prev_to = t_o;
            }
        }
        if (g > 0) issue_pv(prev_first, prev_to);
        if (elect_one()) umma_commit(bars + Lay::B_DRAIN);
        __syncwarp();
        mbar_wait_drain(bars + Lay::B_DRAIN, 0);
    } else {
        // ------------------------------------------------------------ softmax warpgroups
        reg_inc<Lay::SOFTMAX_REGS>();
        const int wg = warp >> 2;
        const int wq = warp & 3;
        const int t = wq * 32 + lane;           // key row of S^T, and d of O^T
        const int q0 = wg * NC;                 // first query column of this warpgroup
        const uint32_t lane_off = (uint32_t)(wq * 32) << 16;
        // this thread's row of the probability tile (128-byte swizzled atoms): its hi and
        // lo columns' 16-byte chunks
        const uint32_t p_row = smem_addr(smem) + Lay::OFF_P +
                               (uint32_t)(t >> 3) * 1024u + (uint32_t)(t & 7) * 128u;
        const uint32_t p_swz = (uint32_t)(t & 7);
        float sl2 = 0.f;          // this tile's scores times it are log2 units: prefix keys come in kKv4Units
        float p_unit = 1.f;       // and the tree's probabilities meet whole values: they go in as units
        float *nm = reinterpret_cast<float *>(smem + Lay::OFF_NM) + q0;           // [NC]
        float *red = reinterpret_cast<float *>(smem + Lay::OFF_RED) + wg * 4 * NC;   // [4][NC]
        float *linv = reinterpret_cast<float *>(smem + Lay::OFF_L) + q0;          // [OB][TP]
        float *pmx = reinterpret_cast<float *>(smem + Lay::OFF_MX) + q0;          // [OB][TP]
        int *parent_s = reinterpret_cast<int *>(smem + Lay::OFF_PARENT) + wg * kMaxTree;

        // the columns' entries of nm, in registers: read by every thread for every tile they were a
        // sixth of shared memory's traffic (a 16-byte load takes four wavefronts, broadcast or not)
        Probs nmr;
        auto load_nm = [&]() {
#pragma unroll
            for (int h = 0; h < NC; h += 4) {
                const ulonglong2 x2 = *reinterpret_cast<const ulonglong2 *>(nm + h);
                nmr[h / 2] = x2.x, nmr[h / 2 + 1] = x2.y;
            }
        };
        uint64_t lacc[NC / 2];   // this key row's share of every owned query's row sum, in pairs
#pragma unroll
        for (int c = 0; c < NC / 2; ++c) lacc[c] = 0ull;
        int g = 0;
        int cur_k = 0;        // this CTA's unit counter (selects the O accumulator)
        // a finished segment whose output still sits in TMEM; a partial one (a
        // unit cut by the work split) goes to its slot instead of the output
        // pend_f: bit 0 a segment is pending, bit 1 it is partial, bit 2 it was
        // the range's first segment, bit 3 its O accumulator
        int pend_f = 0, pend_u = 0, pend_g = 0;

        // The running references lie kKv4Shift below the maxima, which takes the values' unit up
        // again: probabilities are up to 2^20, and one above 2^36 moves its column's reference.
        constexpr float kTooLarge = 6.8719477e10f;
        // Probabilities of this thread's key row for its NC query columns from its raw
        // scores r, against the current running maxima: split into bf16 hi + lo, stored
        // into the probability tile at byte offset `pbuf`, and kept in pr for the row sums.
        // Returns their sum: above kTooLarge (or no number) where one of them is too large, and
        // the exact path then writes the tile again.  (Adding is the FMA pipe's work, a maximum
        // and a split by shifts and masks the integer pipe's, which bounds this loop.)
        auto emit = [&](auto bits_c, const Cols &r, uint32_t bits, uint32_t pbuf, Probs &pr) {
            constexpr bool BITS = decltype(bits_c)::value != 0;
            uint64_t total[2] = {0ull, 0ull};
            const uint64_t sl2x2 = pack2(sl2, sl2);
#pragma unroll
            for (int h = 0; h < NC; h += 8) {
                uint32_t hw[4], lw[4];
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    float d0, d1;
                    unpack2(fma2(pack2(__uint_as_float(r[h + e]), __uint_as_float(r[h + e + 1])), sl2x2, nmr[(h + e) >> 1]),
                            d0, d1);
                    if (BITS) {
                        d0 = ((bits >> (h + e)) & 1u) ? d0 : -INFINITY;
                        d1 = ((bits >> (h + e + 1)) & 1u) ? d1 : -INFINITY;
                    }
                    const uint64_t pp = pack2(ex2(d0), ex2(d1));
                    pr[(h + e) >> 1] = pp;
                    total[(e >> 1) & 1] = add2(total[(e >> 1) & 1], pp);
                    split_bf16x2_fma(BITS ? mul2(pp, pack2(p_unit, p_unit)) : pp, hw[e >> 1], lw[e >> 1]);
                }
                const int ch = q0 + h, cl = TP + q0 + h;   // hi and lo columns
                const uint32_t ah = p_row + pbuf + (uint32_t)(ch >> 6) * Lay::GROUP_BYTES +
                                    ((((uint32_t)(ch & 63) >> 3) ^ p_swz) << 4);
                const uint32_t al = p_row + pbuf + (uint32_t)(cl >> 6) * Lay::GROUP_BYTES +
                                    ((((uint32_t)(cl & 63) >> 3) ^ p_swz) << 4);
                st_shared_v4(ah, hw[0], hw[1], hw[2], hw[3]);
                st_shared_v4(al, lw[0], lw[1], lw[2], lw[3]);
            }
            float s0, s1;
            unpack2(add2(total[0], total[1]), s0, s1);
            return s0 + s1;
        };

        auto load_cols = [&](uint32_t taddr, Cols &r) {   // then tmem_wait_ld
            if constexpr (NC == 32) tmem_ld32(taddr, r);
            else tmem_ld16(taddr, r);
        };

        // A score jumped past its column's maximum by about 2^16: every column's maximum
        // over the 128 key rows is a warp max (redux) combined across the four warps; the row
        // sums, and O unless this is the unit's first tile, are rescaled; the probabilities are
        // computed again, from the scores, which the buffer holds until then.
        auto exact_tile = [&](auto bits_c, uint32_t t_s, uint32_t bits, uint32_t pbuf, bool first, Probs &pr) {
            constexpr bool BITS = decltype(bits_c)::value != 0;
            Cols r;
            load_cols(t_s, r);
            tmem_wait_ld(r);
#pragma unroll
            for (int e = 0; e < NC; ++e) {
                const bool vis = !BITS || ((bits >> e) & 1u) != 0;
                const float mx = warp_max(vis ? __uint_as_float(r[e]) * sl2 : -INFINITY);
                if (lane == e) red[wq * NC + e] = mx;
            }
            named_bar_sync(1 + wg, 128);
            if (t < NC) {
                const float tm = fmaxf(fmaxf(red[t], red[NC + t]), fmaxf(red[2 * NC + t], red[3 * NC + t]));
                const float old = -nm[t];
                const float nw = fmaxf(old, tm - kKv4Shift);
                nm[t] = -nw;
                red[t] = (nw == old) ? 1.f : ex2(old - nw);   // alpha
            }
            named_bar_sync(1 + wg, 128);
            if (!first) {
                // the PV product of the previous tile must have landed first
                mbar_wait(bars + Lay::B_PFREE + ((g - 1) & 1), ((g - 1) >> 1) & 1, abort_flag);
                tc_fence_after();
            }
            const uint32_t t_o = tmem_base + lane_off + Lay::T_O + (uint32_t)(cur_k & 1) * 2 * TP + q0;
#pragma unroll
            for (int h = 0; h < NC; h += 8) {
                float a[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) a[e] = red[h + e];
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    float l0, l1;
                    unpack2(lacc[(h + e) >> 1], l0, l1);
                    lacc[(h + e) >> 1] = pack2(l0 * a[e], l1 * a[e + 1]);
                }
                if (first) continue;   // uniform
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    uint32_t o[8];
                    tmem_ld8(t_o + part * TP + h, o);
                    tmem_wait_ld(o);
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * a[e]);
                    tmem_st8(t_o + part * TP + h, o);
                }
            }
            if (!first) tmem_wait_st();
            load_nm();
            (void)emit(bits_c, r, bits, pbuf, pr);
        };

        // O (hi + lo) of a finished unit's accumulator: one head-dim element per thread,
        // this warpgroup's queries in order, through `put(query column, value)`.
        auto read_o = [&](int ob, int g_last, int n_rows, auto put) {
            mbar_wait(bars + Lay::B_PFREE + (g_last & 1), (g_last >> 1) & 1, abort_flag);
            tc_fence_after();
            if (wq * 32 < D) {
                const uint32_t t_o = tmem_base + lane_off + Lay::T_O + (uint32_t)ob * 2 * TP + q0;
                Cols rh, rl;
                load_cols(t_o, rh);
                load_cols(t_o + TP, rl);
                tmem_wait_ld(rh);
                tmem_wait_ld(rl);
#pragma unroll
                for (int e = 0; e < NC; ++e)
                    if (q0 + e < n_rows) put(e, __uint_as_float(rh[e]) + __uint_as_float(rl[e]));
            }
            tc_fence_before();
        };

        // The pending segment: a whole unit's output times the reciprocal row sums, or the
        // partial state of a cut one into its slot.
        auto flush_pending = [&]() {
            const int ob = (pend_f >> 3) & 1;
            const int lbh = pend_u / p.n_qb, r0 = (pend_u - lbh * p.n_qb) * TP, n_rows = min(TP, R - r0);
            if (!SPLIT || !(pend_f & 2)) {
                const float *li = linv + ob * TP;
                __nv_bfloat16 *orow = reinterpret_cast<__nv_bfloat16 *>(x.out) + ((size_t)lbh * R + r0 + q0) * D + t;
                read_o(ob, pend_g, n_rows, [&](int e, float v) { orow[(size_t)e * D] = __float2bfloat16_rn(v * li[e]); });
            } else {
                float *base = p.split_part + (size_t)(2 * (int)blockIdx.x + ((pend_f & 4) ? 0 : 1)) * kv4_slot_floats(D, TP);
                read_o(ob, pend_g, n_rows, [&](int e, float v) { base[(size_t)(q0 + e) * D + t] = v; });
                if (t < NC && q0 + t < n_rows) {
                    base[(size_t)TP * D + q0 + t] = pmx[ob * TP + t];
                    base[(size_t)TP * D + TP + q0 + t] = linv[ob * TP + t];
                }
            }
        };

        int k = 0;
        UnitIter<SPLIT> it(p, wr);
        for (Seg sg; it.next(p, sg); ++k) {
            const UnitInfo &ui = sg.ui;
            const int u = sg.u;
            cur_k = k;
            const int ob = k & 1;
            if (sg.j1 > ui.n_pref) {   // the sequence's parents, for the tree's tiles
                for (int i = t; i < T; i += 128) cp_async4(smem_addr(parent_s + i), p.parent + (size_t)ui.b * T + i, 4);
                cp_async_commit();
            }
            for (int j = sg.j0; j < sg.j1; ++j, ++g) {
                const bool tree = j >= ui.n_pref;
                const bool first = (j == sg.j0);
                sl2 = tree ? p.scale_log2 : p.scale_log2 * (1.f / kKv4Unit);
                p_unit = tree ? kKv4Unit : 1.f;
                const int n_valid = tree ? Lay::KT : min(Lay::KT, ui.P - j * Lay::KT);
                const bool masked = tree || n_valid < Lay::KT;
                const int sb = g & 1;
                const int ps = g & 1;
                uint32_t dbits = 0;   // bit c: this thread's tree key is visible to row q0 + c
                if (tree) {
                    // lane c walks up from row q0 + c's node and marks its ancestors among the
                    // warp's 32 keys; the 32 x 32 bits turned over, every lane has its key's
                    cp_async_wait<0>();
                    named_bar_sync(1 + wg, 128);
                    const int key0 = (j - ui.n_pref) * Lay::KT + wq * 32, row = ui.qb * TP + q0 + lane;
                    for (int a = lane < NC && row < R ? row % T : -1; a >= key0;) {
                        if (a - key0 < 32) dbits |= 1u << (a - key0);
                        const int up = parent_s[a];
                        a = up < a ? up : -1;   // strictly upwards: ends
                    }
                    __syncwarp();
                    uint32_t m = 0xFFFFu;
#pragma unroll
                    for (int o = 16; o; o >>= 1, m ^= m << o) {
                        const uint32_t y = __shfl_xor_sync(0xffffffffu, dbits, o);
                        dbits = (lane & o) ? (dbits & ~m) | ((y >> o) & m) : (dbits & m) | ((y << o) & ~m);
                    }
                }
                mbar_wait(bars + Lay::B_SFULL + sb, (g >> 1) & 1, abort_flag);
                tc_fence_after();
                const uint32_t t_s = tmem_base + lane_off + Lay::T_S + sb * TP + q0;
                const uint32_t pbuf = (uint32_t)ps * Lay::P_BYTES;
                Cols r;
                load_cols(t_s, r);
                // a probability tile is free once the PV product of tile g - 2 is done
                mbar_wait(bars + Lay::B_PFREE + ps, ((g >> 1) & 1) ^ 1, abort_flag);
                tmem_wait_ld(r);
                if (first) {
                    // a unit starts with the scores of the tile's first key (visible to every
                    // query: a prefix key, or the root) as its maxima: none is above the
                    // true one, and the tile's vote catches any that is too far below.  A part
                    // that starts among the tree's later keys, which not every row sees, takes
                    // the exact path from maxima below every score.
                    if (t == 0) {
                        const bool all_see = j <= ui.n_pref;
#pragma unroll
                        for (int e = 0; e < NC; ++e) nm[e] = all_see ? kKv4Shift - __uint_as_float(r[e]) * sl2 : 1e30f;
                    }
                    named_bar_sync(1 + wg, 128);
                    load_nm();
                }
                // Done optimistically with the current running maxima; when a score
                // exceeds its maximum by more than 2^16, again by the exact path.
                const uint32_t bits = tree ? dbits : (t < n_valid ? 0xffffffffu : 0u);
                Probs pr;
                if (!masked) {
                    const float sum = emit(kind_t<0>{}, r, bits, pbuf, pr);
                    if (named_bar_or(1 + wg, 128, !(sum <= kTooLarge))) exact_tile(kind_t<0>{}, t_s, bits, pbuf, first, pr);
                } else {
                    const float sum = emit(kind_t<1>{}, r, bits, pbuf, pr);
                    if (named_bar_or(1 + wg, 128, !(sum <= kTooLarge))) exact_tile(kind_t<1>{}, t_s, bits, pbuf, first, pr);
                }
                fence_proxy_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bars + Lay::B_PFULL + ps);
#pragma unroll
                for (int c = 0; c < NC / 2; ++c) lacc[c] = add2(lacc[c], pr[c]);

                // the previous segment's output, once this segment's first tile is on its way
                if (first && pend_f) {
                    flush_pending();
                    pend_f = 0;
                }
            }

            // ------------------------------------------ unit end: row sums, LSE
            {
                named_bar_sync(1 + wg, 128);   // every thread is done reading alpha and the maxima
#pragma unroll
                for (int c = 0; c < NC; c += 16) {
                    float v[16];
#pragma unroll
                    for (int e = 0; e < 16; e += 2) unpack2(lacc[(c + e) >> 1], v[e], v[e + 1]);
                    const float s = warp_transpose_reduce16(v, lane, OpAdd());
                    if (!(lane & 1)) red[wq * NC + c + (lane >> 1)] = s;
                }
                named_bar_sync(1 + wg, 128);
                if (t < NC) {
                    const float l = red[t] + red[NC + t] + red[2 * NC + t] + red[3 * NC + t];
                    const float m = -nm[t];
                    if (!SPLIT || seg_whole(sg)) {
                        const int row = ui.qb * TP + q0 + t;
                        if (x.lse && row < R) x.lse[(size_t)ui.lbh * R + row] = (m + lg2(l)) * 0.69314718055994530942f;
                        linv[ob * TP + t] = (1.f / kKv4Unit) / l;
                    } else {
                        linv[ob * TP + t] = l;
                        pmx[ob * TP + t] = m;
                    }
                }
#pragma unroll
                for (int c = 0; c < NC / 2; ++c) lacc[c] = 0ull;
                pend_u = u;
                pend_g = g - 1;
                pend_f = 1 | (ob << 3);
                if (SPLIT && !seg_whole(sg)) {
                    // a part: slot 2c for the range's first segment, 2c + 1 for its last
                    pend_f |= 2 | (sg.u == wr.u_first ? 4 : 0);
                    // the part holding the unit's first tile records it for the merge
                    if (sg.j0 == 0 && threadIdx.x == 0)
                        p.split_rec[blockIdx.x] = SplitRecord{wr.x_first + (wr.n_tiles - it.left) - sg.j1, wr.n_shared, u, ui.n_tiles};
                }
            }
        }
        if (pend_f) {
            named_bar_sync(1 + wg, 128);   // the row sums are in shared memory
            flush_pending();
        }
    }

    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (*abort_flag && threadIdx.x == 0)
        for (int b = 0; b < p.B; ++b) atomicMax(p.dev_status + b, (int)kErrTimeout);
    if (warp == Lay::IW) tmem_dealloc(tmem_base, Lay::TMEM_COLS);
}

// The merge of the units cut by the work split: blockIdx.x is an attention CTA, whose
// record names the unit to merge; a thread merges four columns of a row.
__global__ void __launch_bounds__(256) kv4_wide_merge_kernel(const AttnParams p, const Kv4AttnParams x, int D, int TP)
{
    pdl_release();
    pdl_wait();
    const SplitRecord r = p.split_rec[blockIdx.x];
    if (r.u < 0) return;
    const int per_row = D / 4, G = (int)gridDim.x;
    const int lbh = r.u / p.n_qb, r0 = (r.u - lbh * p.n_qb) * TP, R = x.G * x.T;
    const int row = (int)blockIdx.y * ((int)blockDim.x / per_row) + (int)threadIdx.x / per_row;
    if (row >= min(TP, R - r0)) return;
    const int c0 = ((int)threadIdx.x % per_row) * 4;
    const SplitParts sp = split_parts(r.n_shared, r.off, r.n_tiles);
    const bool dense = r.n_shared >= G;   // no empty ranges
    float M = -INFINITY, L = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c1 = sp.c_a; c1 <= sp.c_b; c1 += 4) {   // four parts' loads in flight
        float m[4], l[4];
        float4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool live = c1 + i <= sp.c_b && (dense || split_nonempty(c1 + i, r.n_shared, G));
            const float *b = p.split_part + (size_t)split_slot(sp, live ? c1 + i : sp.c_a) * kv4_slot_floats(D, TP);
            m[i] = live ? __ldcg(b + (size_t)TP * D + row) : -INFINITY;
            l[i] = __ldcg(b + (size_t)TP * D + TP + row);
            v[i] = __ldcg(reinterpret_cast<const float4 *>(b + (size_t)row * D + c0));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (m[i] == -INFINITY) continue;
            const float nw = fmaxf(M, m[i]), so = ex2(M - nw), w = ex2(m[i] - nw);
            M = nw;
            L = fmaf(L, so, w * l[i]);
            a.x = fmaf(a.x, so, w * v[i].x), a.y = fmaf(a.y, so, w * v[i].y);
            a.z = fmaf(a.z, so, w * v[i].z), a.w = fmaf(a.w, so, w * v[i].w);
        }
    }
    const float inv = (1.f / kKv4Unit) / L;
    const size_t at = (size_t)lbh * R + r0 + row;
    *reinterpret_cast<uint2 *>(x.out + at * D + c0) = make_uint2(bf16x2(a.x * inv, a.y * inv), bf16x2(a.z * inv, a.w * inv));
    if (c0 == 0 && x.lse) x.lse[at] = (M + lg2(L)) * 0.69314718055994530942f;
}

template <int D, int TP, bool SPLIT>
static cudaError_t launch_wide_t(const AttnParams &p, const Kv4AttnParams &x, int grid, cudaStream_t stream)
{
    using Lay = Kv4Wide<D, TP>;
    static std::atomic<uint64_t> configured{0};
    const cudaError_t e = allow_smem(kv4_attention_wide_kernel<D, TP, SPLIT>, Lay::SMEM_BYTES, configured);
    if (e != cudaSuccess) return e;
    return launch_chained_smem(kv4_attention_wide_kernel<D, TP, SPLIT>, dim3((unsigned)grid), dim3(Lay::THREADS), dim3(1), Lay::SMEM_BYTES,
                               stream, p, x);
}

cudaError_t launch_kv4_attention_wide(const AttnParams &p, const Kv4AttnParams &x, int D, int TP, int grid, cudaStream_t stream)
{
    cudaError_t e;
    if (D == 128)
        e = TP == 64 ? (p.split ? launch_wide_t<128, 64, true>(p, x, grid, stream) : launch_wide_t<128, 64, false>(p, x, grid, stream))
                     : (p.split ? launch_wide_t<128, 32, true>(p, x, grid, stream) : launch_wide_t<128, 32, false>(p, x, grid, stream));
    else
        e = TP == 64 ? (p.split ? launch_wide_t<64, 64, true>(p, x, grid, stream) : launch_wide_t<64, 64, false>(p, x, grid, stream))
                     : (p.split ? launch_wide_t<64, 32, true>(p, x, grid, stream) : launch_wide_t<64, 32, false>(p, x, grid, stream));
    if (e != cudaSuccess || !p.split) return e;
    const int rows = 256 / (D / 4);
    return launch_chained(kv4_wide_merge_kernel, dim3((unsigned)grid, (unsigned)((TP + rows - 1) / rows)), dim3(256), dim3(1), stream, p, x, D, TP);
}

}  // namespace ppd
