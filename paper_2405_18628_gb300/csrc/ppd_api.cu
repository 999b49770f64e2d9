// ppd_api.cu -- the C ABI of libppd (declared in include/ppd.h): host-side
// argument checks, workspace layout, TMA tensor-map encoding and the launch
// sequence of each entry point.  No entry point allocates, frees or
// synchronises; all work is enqueued on the caller's stream.
#include "ppd.h"
#include "ppd_kernels.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <atomic>
#include <cstring>
#include <initializer_list>
#include <mutex>

namespace {

using ppd::AcceptArgs;
using ppd::AttnMaps;
using ppd::AttnParams;

constexpr int kMaxT = ppd::kMaxTree;   // tree tokens per sequence
constexpr size_t kAlign = 256;

size_t align_up(size_t x) { return (x + kAlign - 1) & ~(kAlign - 1); }

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// byte ranges [a, a+na) and [b, b+nb) intersect
bool overlaps(const void *a, size_t na, const void *b, size_t nb)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

// Memory that a call reads or writes (null: none).
struct Mem {
    const void *p;
    size_t n;
};

// Blocks of a grid write `out` while others still read `in`: true where an output shares bytes
// with an input or with another output.
bool share_memory(std::initializer_list<Mem> out, std::initializer_list<Mem> in)
{
    for (const Mem *a = out.begin(); a != out.end(); ++a) {
        for (const Mem *b = a + 1; b != out.end(); ++b)
            if (a->p && b->p && overlaps(a->p, a->n, b->p, b->n)) return true;
        for (const Mem &b : in)
            if (a->p && b.p && overlaps(a->p, a->n, b.p, b.n)) return true;
    }
    return false;
}

int num_sms()
{
    static int cache[64] = {0};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
    if (cache[dev] == 0) {
        int n = 0;
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0)
            n = 148;
        cache[dev] = n;
    }
    return cache[dev];
}

int argmax_splits(int64_t rows, int V) { return ppd::argmax_split_count(rows, V); }

// Workspace: the in-grid argmax's sync words, the argmax partials, the side
// warp's scratch, the bf16 copies of fp32 operands, then the work split's
// per-CTA records and partial states.
struct WsLayout {
    size_t part_val, part_idx, part_stats, node_lse, node_ent, side, sync, conv, split_rec,
        split_part, total;
    int splits;
};

int split_grid() { return num_sms() < ppd::kSplitMaxGrid ? num_sms() : ppd::kSplitMaxGrid; }

// Logits per (row, split) chunk of the argmax (a multiple of 4), and whether
// the rows can be read with 16-byte loads; as launch_argmax_partials does.
int argmax_chunk(int V, int splits) { return (((V + splits - 1) / splits) + 3) & ~3; }
int argmax_vec(const float *logits, int V)
{
    return (V % 4 == 0) && ((reinterpret_cast<uintptr_t>(logits) & 15) == 0);
}

// The fused step computes the node argmax inside the attention grid (one
// side warp per CTA, while the other warps stream K/V) when the logits are a
// small share of the bytes the attention streams.  A side warp keeps 2 KB in
// flight (deeper bursts slow the attention more than they gain) and, with the
// HBM saturated by the K/V stream, reads about 1 GB/s against its CTA's
// ~42 GB/s of K/V.  Otherwise a separate argmax grid runs first.  S_max bounds
// the prefix lengths, which only the device knows.  Measured, argmax grid / in-grid:
//   608 slices of 2048 keys, 64 tokens: logits 1/1000 of the K/V bytes 106.3 / 104.2 us,
//     1/100 107.3 / 105.3, 1/64 107.3 / 116.0, 1/50 107.8 / 122.2, 1/20 111.2 / 197.9
//   1216 slices of 4096 keys, 128 tokens: 1/300 356.4 / 352.8, 1/150 357.9 / 356.4,
//     1/100 359.0 / 360.5, 1/64 360.5 / 399.2
//   304 slices of 2048 keys, 200 tokens: 1/300 91.7 / 90.9, 1/64 92.5 / 90.5,
//     1/35 93.0 / 101.2
// With fewer slices than SMs an argmax grid would be shorter at any ratio (32 slices of
// 2048 keys, 1/300: 17.2 / 26.9; 100 at D = 64 19.2 / 22.8): it lets the slices have
// clusters.  The in-grid form shares their tiles out evenly instead, in shorter sums.
constexpr double kInGridMinRatio = 64;
bool in_grid_argmax_pays(int L, int B, int H, int T, int D, int V, int S_max)
{
    const double kv = 4.0 * L * B * H * ((double)S_max + T) * D;
    const double logits = 4.0 * B * (double)T * V;
    return logits * kInGridMinRatio <= kv;
}

// Forms of the fused step (ppd_verify_step_form): separate grids for large
// batches; an argmax grid then the attention grid; one grid whose side warps
// compute the argmax partials while the K/V stream runs.
enum FusedForm { kFormGrids = 0, kFormTwoGrids = 1, kFormSide = 2 };

// A form forced by ppd_set_verify_step_form (-1: chosen by the rules below).
std::atomic<int> g_forced_form{-1};

// The in-grid argmax's grid-wide wait: its limit in ns (0: the default of the
// device-side waits) and a CTA that withholds its flag (-1: none); set only by
// ppd_debug_grid_wait, for tests of the timeout path.
std::atomic<unsigned long long> g_grid_wait_ns{0};
std::atomic<int> g_withhold_cta{-1};

int narrow_argmax_grid(int L, int B, int H, int T, int D, int V, int S_max);

// The form of a fused step (B <= kFusedMaxB) of these sizes: an argmax grid
// first when it fits on the idle SMs of the attention grid's last, partial
// round (measured, us, against the side warps: Vicuna-7B shapes 173.0 / 173.2,
// Vicuna-13B 534.5 / 540.2, MobileLlama 41.3 / 89.9, the batch-8 sweep at 16 tokens
// 9390 / 9397), else the side warps when the logits are a small enough share of the
// K/V bytes, else an argmax grid over every SM.
int choose_form(int L, int B, int H, int T, int D, int V, int S_max)
{
    const int forced = g_forced_form.load(std::memory_order_relaxed);
    if (forced >= kFormTwoGrids) return forced;
    if (narrow_argmax_grid(L, B, H, T, D, V, S_max) > 0) return kFormTwoGrids;
    return in_grid_argmax_pays(L, B, H, T, D, V, S_max) ? kFormSide : kFormTwoGrids;
}

WsLayout workspace_layout(int L, int B, int H, int T, int D, int V, int S_max, ppd_dtype dt)
{
    WsLayout w{};
    const int64_t rows = (int64_t)B * T;
    w.splits = argmax_splits(rows, V);
    size_t off = 0;
    // the in-grid argmax's epoch and all-ready words and per-CTA flags first, at
    // the same offset for every size: a workspace reused for another shape
    // keeps them in place, so its flags only ever hold tags of earlier calls
    w.sync = off;
    off = align_up(off + (size_t)(2 + ppd::kSplitMaxGrid) * 8);
    const size_t cap = (size_t)rows * (size_t)w.splits;
    w.part_val = off;
    off = align_up(off + cap * 4);
    w.part_idx = off;
    off = align_up(off + cap * 4);
    w.part_stats = off;   // softmax statistics partials (typical acceptance)
    off = align_up(off + cap * 12);
    w.node_lse = off;
    off = align_up(off + (size_t)rows * 4);
    w.node_ent = off;
    off = align_up(off + (size_t)rows * 4);
    w.side = off;
    off = align_up(off + (size_t)num_sms() * ppd::kSideScratchInts * 4);
    w.conv = off;
    if (dt == PPD_F32) {
        const size_t lbh = (size_t)L * B * H;
        off = align_up(off + lbh * ((size_t)3 * T + 2 * (size_t)S_max) * D * 2);
    }
    w.split_rec = off;
    off = align_up(off + (size_t)split_grid() * sizeof(ppd::SplitRecord));
    w.split_part = off;
    off = align_up(off + (size_t)2 * split_grid() * ppd::kSplitRows * (D + 2) * sizeof(float));
    w.total = off;
    return w;
}

// ------------------------------------------------------------------ tensor maps

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                                  const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                  const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn()
{
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                             &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    });
    return fn;
}

// bf16 tensor viewed as [depth][rows][inner], box {64, box_rows, 1}, 128-byte swizzle,
// out-of-range rows read as zero.
bool encode_3d(CUtensorMap *m, const void *base, uint64_t inner, uint64_t rows, uint64_t depth,
               uint32_t box_rows)
{
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    const cuuint64_t dims[3] = {inner, rows, depth};
    const cuuint64_t strides[2] = {inner * 2, inner * 2 * rows};
    const cuuint32_t box[3] = {64, box_rows, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box,
               estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool encode_2d(CUtensorMap *m, const void *base, uint64_t inner, uint64_t rows, uint32_t box_rows)
{
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    const cuuint64_t dims[2] = {inner, rows};
    const cuuint64_t strides[1] = {inner * 2};
    const cuuint32_t box[2] = {64, box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, strides, box,
               estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The CUDA error behind the latest PPD_ERR_CUDA of this process (diagnostics).
std::atomic<int> g_last_cuda_error{cudaSuccess};

// A launch reported failed through the runtime's last error (kernels launched
// with <<< >>>): record it and clear it.
ppd_status cuda_failed()
{
    const cudaError_t e = cudaGetLastError();
    g_last_cuda_error.store((int)(e != cudaSuccess ? e : cudaErrorUnknown), std::memory_order_relaxed);
    return PPD_ERR_CUDA;
}

// A failed call clears the runtime's last-error state (errors that do not
// break the context), so it cannot surface as the status of a later call.
ppd_status cuda_status(cudaError_t e)
{
    if (e == cudaSuccess) return PPD_OK;
    g_last_cuda_error.store((int)e, std::memory_order_relaxed);
    (void)cudaGetLastError();
    return PPD_ERR_CUDA;
}

// ------------------------------------------------------------------ shared checks

bool attn_dims_ok(int L, int B, int H, int T, int D, int S_max, ppd_dtype dt)
{
    if (L < 1 || B < 1 || H < 1 || T < 1 || T > kMaxT || S_max < 1) return false;
    if (D != 64 && D != 128) return false;
    if (dt != PPD_BF16 && dt != PPD_F32) return false;
    const double lbh = (double)L * B * H;
    if (lbh > 2147483647.0 || lbh * S_max * D > 9.0e15) return false;
    return true;
}

// How an attention launch shares its work out: whole units round-robin, one
// cluster of CTAs per unit (cluster > 1), or equal ranges of all key tiles
// (split; needs a workspace and a batch of at most kSplitMaxB).  Only launches
// with fewer units than SMs can gain from either: with more, the last round's
// idle SMs cost less than the merge (measured on the Vicuna-7B/13B and
// MobileLlama shapes).  Counted in tiles of 128 keys, S_max standing in for the
// (device-side) prefix lengths: whole units take t_u tiles; a cluster of c takes
// its share and about kClusterCostTiles for the merge through distributed
// shared memory; the work split takes its share of all tiles, which is smaller,
// and about kSplitCostTiles for the range planning and the merge grid.  Measured per
// call, D = 128, 64 tokens, whole / split / cluster:
//   20 units of 4 tiles  8.6 / 11.7 /  8.1 us     32 of 13  16.6 / 17.8 / 12.7
//   60 of 7             11.9 / 18.1 / 12.7        48 of 25  28.0 / 25.5 / 21.5
//   80 of 25            31.3 / 33.5               80 of 64  69.0 / 63.1
//   100 of 25           32.8 / 39.0               20 of 64  61.5 / 27.0 / 21.0
// By the time alone the split would cost sixteen tiles (10 us for planning and merging,
// and longer tiles with every SM streaming) and a cluster three or four.  The lines are
// not drawn there: parts keep the fp32 sums short, and the calls that would change over
// lose that (relative error against 64 bits with the split at sixteen: 100 units of 25
// tiles 3.1e-6 -> 4.2e-6, 120 of 64 6.2e-6 -> 9.5e-6, 48 of 64 3.6e-6 -> 5.2e-6).
struct AttnPlan {
    int split, cluster;
};
constexpr long long kClusterCostTiles = 2, kSplitCostTiles = 6;

AttnPlan plan_attention(int L, int B, int H, int T, int S_max, bool workspace, bool clusters)
{
    AttnPlan plan{0, 1};
    const int n_tt = T > 64 ? (T + 127) / 128 : 1;
    const long long units = (long long)L * B * H * n_tt, sms = split_grid();
    if (units >= sms) return plan;
    const long long t_u = (S_max + 127) / 128 + n_tt;
    long long best = t_u;
    for (int c = 2; clusters && c <= ppd::kMaxCluster && c <= t_u && units * c <= sms; ++c) {
        const long long cost = (t_u + c - 1) / c + kClusterCostTiles;
        if (cost < best && units <= ppd::max_attention_clusters(c)) {
            best = cost;
            plan.cluster = c;
        }
    }
    if (workspace && B <= ppd::kSplitMaxB && (units * t_u + sms - 1) / sms + kSplitCostTiles < best) plan = {1, 1};
    return plan;
}

// Enqueue the attention of all L*B*H slices (bf16 operands).
// set_status: every sequence's dev_status is written (else only raised).
ppd_status enqueue_attention(const void *q, const void *kc, const void *vc, const void *kt,
                             const void *vt, const int32_t *prefix_len, const int32_t *parent,
                             int L, int B, int H, int T, int D, int S_max, float scale, float *out,
                             float *lse, int32_t *dev_status, uint8_t *ws, const WsLayout *wl,
                             const ppd::FusedStep *fused, bool programmatic, bool chained,
                             bool set_status, cudaStream_t stream)
{
    const int T_pad = (T + 31) & ~31;
    const uint64_t lbh = (uint64_t)L * B * H;
    // trees of more than 64 tokens run the row-layout kernel, which reads Q in
    // boxes of 128 rows (rows past T arrive as zeros)
    const uint32_t q_box = T_pad > 64 ? 128u : (uint32_t)T_pad;
    AttnMaps m;
    if (!encode_3d(&m.q, q, D, T, lbh, q_box) || !encode_3d(&m.kc, kc, D, S_max, lbh, 128) ||
        !encode_3d(&m.vc, vc, D, S_max, lbh, 128) || !encode_3d(&m.kt, kt, D, T, lbh, 128) ||
        !encode_3d(&m.vt, vt, D, T, lbh, 128))
        return PPD_ERR_CUDA;
    AttnParams p{};
    p.prefix_len = prefix_len;
    p.parent = parent;
    p.out = out;
    p.lse = lse;
    p.dev_status = dev_status;
    p.L = L;
    p.B = B;
    p.H = H;
    p.T = T;
    p.T_pad = T_pad;
    p.S_max = S_max;
    // trees of more than 64 tokens: slices split into blocks of 128 query rows,
    // the tree keys into tiles of 128
    p.n_qb = T_pad > 64 ? (T + 127) / 128 : 1;
    p.n_tt = T_pad > 64 ? (T + 127) / 128 : 1;
    p.n_units = (int)lbh * p.n_qb;
    const float sc = scale > 0.f ? scale : 1.0f / std::sqrt((float)D);
    p.scale_log2 = sc * 1.4426950408889634f;
    ppd::plan_rows(p, split_grid());
    const AttnPlan plan = plan_attention(L, B, H, T, S_max, ws && wl, !(fused && fused->in_grid));
    p.cluster = plan.cluster;
    p.set_status = set_status;
    if (plan.split) {
        p.split = 1;
        p.split_rec = reinterpret_cast<ppd::SplitRecord *>(ws + wl->split_rec);
        p.split_part = reinterpret_cast<float *>(ws + wl->split_part);
    }
    p.fused = fused != nullptr;
    if (fused) p.fs = *fused;
    p.pdl_wait = chained ? 1 : 0;
    p.late_wait = programmatic && !chained && !fused ? 1 : 0;
    return cuda_status(ppd::launch_tree_attention(m, p, D, split_grid(), programmatic || chained,
                                                  stream));
}

// fp32 operands: round to bf16 copies in the workspace first (of the caches the
// rows below each prefix): by five grids, as the fused step counts them, or
// (chained) by one in the chain of programmatic launches.  chained: the call is a
// link of such a chain and its attention grid waits for whatever precedes it
// itself.  A fused step's bf16 attention grid overlaps the argmax grid before it
// -- when there is one: it only reads caller inputs before its end phase.
ppd_status enqueue_attention_any(const void *q, const void *kc, const void *vc, const void *kt,
                                 const void *vt, const int32_t *prefix_len, const int32_t *parent,
                                 int L, int B, int H, int T, int D, int S_max, ppd_dtype dt,
                                 float scale, float *out, float *lse, int32_t *dev_status,
                                 uint8_t *ws, const WsLayout &wl, const ppd::FusedStep *fused,
                                 cudaStream_t stream, bool chained = false)
{
    if (dt == PPD_BF16)
        return enqueue_attention(q, kc, vc, kt, vt, prefix_len, parent, L, B, H, T, D, S_max, scale,
                                 out, lse, dev_status, ws, ws ? &wl : nullptr, fused,
                                 fused != nullptr && !fused->in_grid, chained, chained, stream);
    const int64_t lbh = (int64_t)L * B * H;
    const int64_t n_t = lbh * T * D, n_c = lbh * (int64_t)S_max * D;
    uint16_t *bq = reinterpret_cast<uint16_t *>(ws + wl.conv);
    uint16_t *bkt = bq + n_t;
    uint16_t *bvt = bkt + n_t;
    uint16_t *bkc = bvt + n_t;
    uint16_t *bvc = bkc + n_c;
    ppd::RoundArgs r{};
    const void *src[5] = {q, kt, vt, kc, vc};
    uint16_t *dst[5] = {bq, bkt, bvt, bkc, bvc};
    r.prefix_len = prefix_len;
    r.B = B;
    r.H = H;
    r.D = D;
    for (int i = 0; i < 5; ++i) r.t[i] = {(const float *)src[i], dst[i], i < 3 ? T : S_max, i >= 3};
    if (chained) {
        r.n = 5;
        const cudaError_t e = ppd::launch_round_bf16(r, lbh, true, stream);
        if (e != cudaSuccess) return cuda_status(e);
    } else {
        for (int i = 0; i < 5; ++i) {
            ppd::RoundArgs one = r;
            one.t[0] = r.t[i];
            one.n = 1;
            const cudaError_t e = ppd::launch_round_bf16(one, lbh, false, stream);
            if (e != cudaSuccess) return cuda_status(e);
        }
    }
    return enqueue_attention(bq, bkc, bvc, bkt, bvt, prefix_len, parent, L, B, H, T, D, S_max,
                             scale, out, lse, dev_status, ws, &wl, fused, false, chained, chained, stream);
}

// The jobs of an attention launch without a split: its units, with plan_rows' choice.
AttnParams row_plan(int L, int B, int H, int T, int S_max)
{
    AttnParams p{};
    p.T_pad = (T + 31) & ~31;
    p.n_qb = p.T_pad > 64 ? (T + 127) / 128 : 1;
    p.n_units = (int)((long long)L * B * H) * p.n_qb;
    p.S_max = S_max;
    ppd::plan_rows(p, split_grid());
    return p;
}

// Blocks of the fused step's narrow argmax grid (0: use the wide grid).  When
// the attention grid's jobs do not fill whole rounds, the CTAs of the last,
// partial round that hold one job fewer -- grid - (jobs mod grid) of
// them -- have a slice's time to spare; the argmax blocks take as many SMs
// (at most half of them), the CTAs dispatched last, which are those, wait for
// them, and nothing on the critical path does.  Each block's share of the
// logits must then be at most half a slice's K/V bytes (S_max standing in for
// the device-side prefix lengths).  Either split (fewer slices than SMs) leaves
// no CTA with time to spare.
int narrow_argmax_grid(int L, int B, int H, int T, int D, int V, int S_max)
{
    const AttnPlan plan = plan_attention(L, B, H, T, S_max, true, true);
    if (plan.split || plan.cluster > 1) return 0;
    const AttnParams p = row_plan(L, B, H, T, S_max);
    // two groups of CTAs with queues of their own: none is known to have time to spare
    if (p.pairs && p.n_qb == 3) return 0;
    const long long n_jobs = ppd::whole_jobs(p);
    const long long grid = ppd::attention_grid(p, split_grid());
    const long long r = n_jobs % grid;
    if (r == 0) return 0;
    long long g = grid - r;
    if (g > num_sms() / 2) g = num_sms() / 2;
    if (g < 8) return 0;
    const double logits = 4.0 * B * (double)T * V;
    const double slice = 4.0 * ((double)S_max + T) * D;
    return logits / (double)g <= slice / 2 ? (int)g : 0;
}

}  // namespace

// Parameters of typical acceptance (null: exact matching).
struct TypicalParams {
    float temperature, epsilon, delta;
};

static ppd_status verify_step_impl(const void *q, void *k_cache, void *v_cache,
                                   const void *k_tree, const void *v_tree,
                                   const int32_t *prefix_len, const int32_t *parent,
                                   const int32_t *cand_tokens, const float *logits, int L, int B,
                                   int H, int T, int D, int V, int S_max, ppd_dtype dt, float scale,
                                   const TypicalParams *typ, float *out, float *lse,
                                   int32_t *argmax_out, int32_t *accept_len, int32_t *path,
                                   int32_t *next_token, int32_t *new_prefix_len,
                                   int32_t *dev_status, void *workspace, size_t ws_bytes,
                                   void *stream)
{
    if (!q || !k_cache || !v_cache || !k_tree || !v_tree || !prefix_len || !parent ||
        !cand_tokens || !logits || !out || !argmax_out || !accept_len || !path || !next_token ||
        !new_prefix_len || !dev_status || !workspace)
        return PPD_ERR_INVALID_ARG;
    if (!attn_dims_ok(L, B, H, T, D, S_max, dt) || V < 1 || !std::isfinite(scale))
        return PPD_ERR_INVALID_ARG;
    if ((double)B * T * V > 9.0e15) return PPD_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(k_tree, 16) ||
        !aligned(v_tree, 16) || !aligned(out, 4) || !aligned(lse, 4))
        return PPD_ERR_INVALID_ARG;
    const int eb = dt == PPD_BF16 ? 2 : 4;
    const size_t lbh = (size_t)L * B * H;
    const size_t nc = lbh * S_max * D * eb, nt = lbh * T * D * eb;
    if (overlaps(k_cache, nc, k_tree, nt) || overlaps(k_cache, nc, v_tree, nt) ||
        overlaps(v_cache, nc, k_tree, nt) || overlaps(v_cache, nc, v_tree, nt) ||
        overlaps(k_cache, nc, v_cache, nc))
        return PPD_ERR_INVALID_ARG;
    const WsLayout wl = workspace_layout(L, B, H, T, D, V, S_max, dt);
    if (ws_bytes < wl.total || !aligned(workspace, kAlign)) return PPD_ERR_INVALID_ARG;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    float *pv = reinterpret_cast<float *>(ws + wl.part_val);
    int32_t *pi = reinterpret_cast<int32_t *>(ws + wl.part_idx);
    float *pst = typ ? reinterpret_cast<float *>(ws + wl.part_stats) : nullptr;
    const float temp = typ ? typ->temperature : 1.f;
    const int64_t rows = (int64_t)B * T;

    if (B <= ppd::kFusedMaxB) {
        bool in_grid = choose_form(L, B, H, T, D, V, S_max) == kFormSide;
        while (true) {
            // 1. partial maxima (and statistics) of every node's logits; also zeroes
            //    dev_status.  In-grid: the attention grid's side warps do this instead.
            if (!in_grid) {
                const int narrow = narrow_argmax_grid(L, B, H, T, D, V, S_max);
                const cudaError_t e =
                    narrow > 0 ? ppd::launch_argmax_narrow(logits, rows, V, wl.splits, narrow, pv, pi, pst,
                                                           temp, dev_status, B, s)
                               : ppd::launch_argmax_partials(logits, rows, V, wl.splits, pv, pi, pst, temp,
                                                             dev_status, B, s);
                if (e != cudaSuccess) return cuda_status(e);
            }
            // 2. attention over every layer, overlapping step 1; its side warps combine
            //    the argmax, decide acceptance and compact the accepted rows
            ppd::FusedStep f{};
            f.part_val = pv;
            f.part_idx = pi;
            f.splits = wl.splits;
            f.cand_tokens = cand_tokens;
            f.argmax_out = argmax_out;
            f.accept_len = accept_len;
            f.path = path;
            f.next_token = next_token;
            f.new_prefix_len = new_prefix_len;
            f.status = dev_status;
            f.k_cache = static_cast<uint8_t *>(k_cache);
            f.v_cache = static_cast<uint8_t *>(v_cache);
            f.k_tree = static_cast<const uint8_t *>(k_tree);
            f.v_tree = static_cast<const uint8_t *>(v_tree);
            f.row_bytes = D * eb;
            f.V = V;
            f.scratch = reinterpret_cast<int *>(ws + wl.side);
            f.logits = logits;
            if (in_grid) {
                f.in_grid = 1;
                f.chunk = argmax_chunk(V, wl.splits);
            }
            if (in_grid) {
                // no argmax grid to zero the status first: a one-block reset does,
                // so that every status write can be an atomic maximum
                if (ppd::launch_zero_status(dev_status, B, s) != cudaSuccess) return cuda_failed();
                const unsigned long long lim = g_grid_wait_ns.load(std::memory_order_relaxed);
                f.wait_limit_ns = lim ? lim : ppd::kWaitLimitNs;
                f.withhold_cta = g_withhold_cta.load(std::memory_order_relaxed);
                f.vec = argmax_vec(logits, V);
                f.stat_k = 1.4426950408889634f / temp;
                f.epoch = reinterpret_cast<unsigned long long *>(ws + wl.sync);
                f.all_ready = f.epoch + 1;
                f.ready = f.epoch + 2;
            }
            if (typ) {
                f.typical = 1;
                f.part_stats = pst;
                f.inv_temp = 1.f / typ->temperature;
                f.epsilon = typ->epsilon;
                f.delta = typ->delta;
            }
            const ppd_status st = enqueue_attention_any(q, k_cache, v_cache, k_tree, v_tree,
                                                        prefix_len, parent, L, B, H, T, D, S_max,
                                                        dt, scale, out, lse, nullptr, ws, wl, &f, s);
            if (st == PPD_OK || !in_grid) return st;
            // the cooperative launch could not have every CTA resident (SMs taken by
            // other work): clear its error and run the argmax as its own grid
            if (g_last_cuda_error.load(std::memory_order_relaxed) != cudaErrorCooperativeLaunchTooLarge)
                return st;
            in_grid = false;
        }
    }

    // large batches: the same steps as separate grids, the combine, the acceptance and
    // (bf16) the attention grid as a chain of programmatic launches: the attention reads
    // nothing that this step's other grids write, so it starts where the first grid's
    // blocks leave the SMs (80 sequences: 250 -> 242 us); one of its warps waits for them
    AcceptArgs a{cand_tokens, parent, prefix_len, accept_len, path, next_token, new_prefix_len,
                 dev_status, T, V, S_max};
    if (ppd::launch_argmax_partials(logits, rows, V, wl.splits, pv, pi, pst, temp, nullptr, 0, s) !=
        cudaSuccess)
        return cuda_failed();
    cudaError_t e;
    if (typ) {
        float *nl = reinterpret_cast<float *>(ws + wl.node_lse);
        float *ne = reinterpret_cast<float *>(ws + wl.node_ent);
        e = ppd::launch_node_stats_combine(pv, pi, pst, rows, wl.splits, argmax_out, nl, ne, s);
        if (e == cudaSuccess)
            e = ppd::launch_typical_accept(logits, nl, ne, argmax_out, a, B, typ->temperature, typ->epsilon,
                                           typ->delta, s);
    } else {
        e = ppd::launch_argmax_combine(pv, pi, rows, wl.splits, argmax_out, s);
        if (e == cudaSuccess) e = ppd::launch_accept_path(argmax_out, a, B, s);
    }
    if (e != cudaSuccess) return cuda_status(e);
    ppd_status st;
    if (dt == PPD_BF16)
        st = enqueue_attention(q, k_cache, v_cache, k_tree, v_tree, prefix_len, parent, L, B, H, T, D, S_max,
                               scale, out, lse, dev_status, ws, &wl, nullptr, true, false, false, s);
    else
        st = enqueue_attention_any(q, k_cache, v_cache, k_tree, v_tree, prefix_len, parent, L, B, H, T, D,
                                   S_max, dt, scale, out, lse, dev_status, ws, wl, nullptr, s);
    if (st != PPD_OK) return st;
    // in plain stream order: it needs the attention done, which waited for the acceptance
    return cuda_status(ppd::launch_kv_compact(k_cache, v_cache, k_tree, v_tree, path, accept_len,
                                              prefix_len, L, B, H, T, D, S_max, eb, s, false));
}

int ppd_verify_step_form(int L, int B, int H, int T, int D, int V, int S_max, ppd_dtype dt)
{
    if (!attn_dims_ok(L, B, H, T, D, S_max, dt) || V < 1) return -1;
    if (B > ppd::kFusedMaxB) return kFormGrids;
    return choose_form(L, B, H, T, D, V, S_max);
}

int ppd_attention_plan(int L, int B, int H, int T, int D, int S_max, int workspace, int one_grid)
{
    if (!attn_dims_ok(L, B, H, T, D, S_max, PPD_BF16)) return -1;
    const AttnPlan plan = plan_attention(L, B, H, T, S_max, workspace != 0, one_grid == 0);
    if (plan.split || plan.cluster > 1) return plan.split ? 1 : plan.cluster;
    return row_plan(L, B, H, T, S_max).pairs ? 16 : 0;
}

ppd_status ppd_debug_grid_wait(unsigned long long limit_ns, int withhold_cta)
{
    if (withhold_cta < -1) return PPD_ERR_INVALID_ARG;
    g_grid_wait_ns.store(limit_ns);
    g_withhold_cta.store(withhold_cta);
    return PPD_OK;
}

int ppd_set_verify_step_form(int form)
{
    if (form != -1 && form != kFormTwoGrids && form != kFormSide) return -2;
    return g_forced_form.exchange(form);
}

int ppd_verify_step_launches(int L, int B, int H, int T, int D, int V, int S_max, ppd_dtype dt,
                             int typical)
{
    (void)typical;   // both acceptance rules launch the same number of kernels
    const int form = ppd_verify_step_form(L, B, H, T, D, V, S_max, dt);
    if (form < 0) return -1;
    const int round = dt == PPD_F32 ? 5 : 0;   // fp32 -> bf16 copies of Q, K/V tree, K/V cache
    const int attn = plan_attention(L, B, H, T, S_max, true, form != kFormSide).split ? 2 : 1;   // + the merge grid
    if (form == kFormTwoGrids) return 1 + round + attn;
    if (form == kFormSide) return 1 + round + attn;   // the status reset, then one grid
    // partial maxima, combine (or statistics), acceptance, attention, compaction
    return 3 + round + attn + 1;
}

static bool typical_params_ok(float temperature, float epsilon, float delta)
{
    return std::isfinite(temperature) && temperature > 0.f && std::isfinite(epsilon) &&
           std::isfinite(delta) && std::isfinite(1.f / temperature);
}

extern "C" {

size_t ppd_workspace_bytes(int L, int B, int H, int T, int D, int V, int S_max, ppd_dtype dt)
{
    if (L < 1 || B < 1 || H < 1 || T < 1 || D < 1 || V < 1 || S_max < 0) return 0;
    return workspace_layout(L, B, H, T, D, V, S_max, dt).total;
}


const char *ppd_last_cuda_error(void)
{
    return cudaGetErrorName((cudaError_t)g_last_cuda_error.load(std::memory_order_relaxed));
}

const char *ppd_status_string(ppd_status s)
{
    switch (s) {
    case PPD_OK: return "ok";
    case PPD_ERR_INVALID_ARG: return "invalid argument";
    case PPD_ERR_UNSUPPORTED: return "unsupported configuration";
    case PPD_ERR_TREE: return "malformed tree or token id";
    case PPD_ERR_CAPACITY: return "cache capacity exceeded or prefix length out of range";
    case PPD_ERR_CUDA: return "CUDA runtime error";
    case PPD_ERR_TIMEOUT: return "device-side wait timed out";
    }
    return "unknown status";
}

ppd_status ppd_tree_attention(const void *q, const void *k_cache, const void *v_cache,
                              const void *k_tree, const void *v_tree,
                              const int32_t *prefix_len, const int32_t *parent,
                              int L, int B, int H, int T, int D, int S_max, ppd_dtype dt,
                              float scale, float *out, float *lse, int32_t *dev_status,
                              void *workspace, size_t ws_bytes, void *stream)
{
    if (!q || !k_cache || !v_cache || !k_tree || !v_tree || !prefix_len || !parent || !out ||
        !dev_status)
        return PPD_ERR_INVALID_ARG;
    if (!attn_dims_ok(L, B, H, T, D, S_max, dt) || !std::isfinite(scale)) return PPD_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(k_tree, 16) ||
        !aligned(v_tree, 16) || !aligned(out, 4) || !aligned(lse, 4))
        return PPD_ERR_INVALID_ARG;
    const WsLayout wl = workspace_layout(L, B, H, T, D, 1, S_max, dt);
    const bool ws_ok = workspace && ws_bytes >= wl.total && aligned(workspace, kAlign);
    if (dt == PPD_F32 && !ws_ok) return PPD_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // one link of a chain of programmatic launches (one call per layer, as a model
    // runs them): the grid starts while the previous one still runs, does the setup
    // that reads no input, and waits for it; its spare warps write dev_status
    // (a bf16 call without a full workspace has no work split)
    return enqueue_attention_any(q, k_cache, v_cache, k_tree, v_tree, prefix_len, parent, L, B, H,
                                 T, D, S_max, dt, scale, out, lse, dev_status,
                                 ws_ok ? static_cast<uint8_t *>(workspace) : nullptr, wl, nullptr, s,
                                 true);
}

ppd_status ppd_node_argmax(const float *logits, int B, int T, int V, int32_t *argmax_out,
                           void *workspace, size_t ws_bytes, void *stream)
{
    if (!logits || !argmax_out || B < 1 || T < 1 || V < 1) return PPD_ERR_INVALID_ARG;
    if ((double)B * T * V > 9.0e15 || (double)B * T * 64 > 2147483647.0) return PPD_ERR_INVALID_ARG;
    const WsLayout wl = workspace_layout(1, B, 1, T, 1, V, 0, PPD_BF16);
    if (!workspace || ws_bytes < wl.total || !aligned(workspace, kAlign)) return PPD_ERR_INVALID_ARG;
    return cuda_status(ppd::launch_node_argmax(logits, (int64_t)B * T, V, 1.f, argmax_out, nullptr, nullptr,
                                               static_cast<cudaStream_t>(stream)));
}

// The same grid as ppd_node_argmax, which needs no scratch; requests of more than
// 65,536 rows stay refused.
ppd_status ppd_node_argmax_noalloc(const float *logits, int B, int T, int V, int32_t *argmax_out, void *stream)
{
    constexpr int64_t kMaxRows = 1 << 16;
    if (!logits || !argmax_out || B < 1 || T < 1 || V < 1) return PPD_ERR_INVALID_ARG;
    if ((double)B * T * V > 9.0e15) return PPD_ERR_INVALID_ARG;
    const int64_t rows = (int64_t)B * T;
    if (rows > kMaxRows) return PPD_ERR_UNSUPPORTED;
    return cuda_status(ppd::launch_node_argmax(logits, rows, V, 1.f, argmax_out, nullptr, nullptr,
                                               static_cast<cudaStream_t>(stream)));
}

ppd_status ppd_accept_path(const int32_t *argmax, const int32_t *cand_tokens,
                           const int32_t *parent, const int32_t *prefix_len,
                           int B, int T, int V, int S_max,
                           int32_t *accept_len, int32_t *path, int32_t *next_token,
                           int32_t *new_prefix_len, int32_t *dev_status, void *stream)
{
    if (!argmax || !cand_tokens || !parent || !prefix_len || !accept_len || !path || !next_token ||
        !new_prefix_len || !dev_status)
        return PPD_ERR_INVALID_ARG;
    if (B < 1 || T < 1 || T > kMaxT || V < 1 || S_max < 0) return PPD_ERR_INVALID_ARG;
    AcceptArgs a{cand_tokens, parent, prefix_len, accept_len, path, next_token, new_prefix_len,
                 dev_status, T, V, S_max};
    return cuda_status(ppd::launch_accept_path(argmax, a, B, static_cast<cudaStream_t>(stream)));
}

ppd_status ppd_kv_compact(void *k_cache, void *v_cache, const void *k_tree, const void *v_tree,
                          const int32_t *path, const int32_t *accept_len,
                          const int32_t *prefix_len, int L, int B, int H, int T, int D,
                          int S_max, ppd_dtype dt, void *stream)
{
    if (!k_cache || !v_cache || !k_tree || !v_tree || !path || !accept_len || !prefix_len)
        return PPD_ERR_INVALID_ARG;
    if (L < 1 || B < 1 || H < 1 || T < 1 || T > kMaxT || D < 1 || S_max < 0) return PPD_ERR_INVALID_ARG;
    if (dt != PPD_BF16 && dt != PPD_F32) return PPD_ERR_INVALID_ARG;
    const int eb = dt == PPD_BF16 ? 2 : 4;
    if ((D * eb) % 16 != 0) return PPD_ERR_UNSUPPORTED;
    if (!aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(k_tree, 16) || !aligned(v_tree, 16))
        return PPD_ERR_INVALID_ARG;
    const size_t lbh = (size_t)L * B * H;
    const size_t nc = lbh * S_max * D * eb, nt = lbh * T * D * eb;
    if (overlaps(k_cache, nc, k_tree, nt) || overlaps(k_cache, nc, v_tree, nt) ||
        overlaps(v_cache, nc, k_tree, nt) || overlaps(v_cache, nc, v_tree, nt) ||
        overlaps(k_cache, nc, v_cache, nc))
        return PPD_ERR_INVALID_ARG;
    return cuda_status(ppd::launch_kv_compact(k_cache, v_cache, k_tree, v_tree, path, accept_len,
                                              prefix_len, L, B, H, T, D, S_max, eb,
                                              static_cast<cudaStream_t>(stream)));
}

ppd_status ppd_verify_step(const void *q, void *k_cache, void *v_cache,
                           const void *k_tree, const void *v_tree,
                           const int32_t *prefix_len, const int32_t *parent,
                           const int32_t *cand_tokens, const float *logits,
                           int L, int B, int H, int T, int D, int V, int S_max, ppd_dtype dt,
                           float scale, float *out, float *lse, int32_t *argmax_out,
                           int32_t *accept_len, int32_t *path, int32_t *next_token,
                           int32_t *new_prefix_len, int32_t *dev_status,
                           void *workspace, size_t ws_bytes, void *stream)
{
    return verify_step_impl(q, k_cache, v_cache, k_tree, v_tree, prefix_len, parent, cand_tokens,
                            logits, L, B, H, T, D, V, S_max, dt, scale, nullptr, out, lse,
                            argmax_out, accept_len, path, next_token, new_prefix_len, dev_status,
                            workspace, ws_bytes, stream);
}

ppd_status ppd_verify_step_typical(const void *q, void *k_cache, void *v_cache,
                                   const void *k_tree, const void *v_tree,
                                   const int32_t *prefix_len, const int32_t *parent,
                                   const int32_t *cand_tokens, const float *logits,
                                   int L, int B, int H, int T, int D, int V, int S_max,
                                   ppd_dtype dt, float scale, float temperature, float epsilon,
                                   float delta, float *out, float *lse, int32_t *argmax_out,
                                   int32_t *accept_len, int32_t *path, int32_t *next_token,
                                   int32_t *new_prefix_len, int32_t *dev_status,
                                   void *workspace, size_t ws_bytes, void *stream)
{
    if (!typical_params_ok(temperature, epsilon, delta)) return PPD_ERR_INVALID_ARG;
    const TypicalParams typ{temperature, epsilon, delta};
    return verify_step_impl(q, k_cache, v_cache, k_tree, v_tree, prefix_len, parent, cand_tokens,
                            logits, L, B, H, T, D, V, S_max, dt, scale, &typ, out, lse,
                            argmax_out, accept_len, path, next_token, new_prefix_len, dev_status,
                            workspace, ws_bytes, stream);
}

ppd_status ppd_node_stats(const float *logits, int B, int T, int V, float temperature,
                          int32_t *argmax_out, float *lse_out, float *entropy_out,
                          void *workspace, size_t ws_bytes, void *stream)
{
    if (!logits || !argmax_out || !lse_out || !entropy_out || B < 1 || T < 1 || V < 1)
        return PPD_ERR_INVALID_ARG;
    if (!std::isfinite(temperature) || !(temperature > 0.f) || !std::isfinite(1.f / temperature))
        return PPD_ERR_INVALID_ARG;
    if ((double)B * T * V > 9.0e15 || (double)B * T * 64 > 2147483647.0) return PPD_ERR_INVALID_ARG;
    const WsLayout wl = workspace_layout(1, B, 1, T, 1, V, 0, PPD_BF16);
    if (!workspace || ws_bytes < wl.total || !aligned(workspace, kAlign)) return PPD_ERR_INVALID_ARG;
    return cuda_status(ppd::launch_node_argmax(logits, (int64_t)B * T, V, temperature, argmax_out, lse_out,
                                               entropy_out, static_cast<cudaStream_t>(stream)));
}

ppd_status ppd_typical_accept(const float *logits, const float *lse, const float *entropy,
                              const int32_t *argmax, const int32_t *cand_tokens,
                              const int32_t *parent, const int32_t *prefix_len, int B, int T,
                              int V, int S_max, float temperature, float epsilon, float delta,
                              int32_t *accept_len, int32_t *path, int32_t *next_token,
                              int32_t *new_prefix_len, int32_t *dev_status, void *stream)
{
    if (!logits || !lse || !entropy || !argmax || !cand_tokens || !parent || !prefix_len ||
        !accept_len || !path || !next_token || !new_prefix_len || !dev_status)
        return PPD_ERR_INVALID_ARG;
    if (B < 1 || T < 1 || T > kMaxT || V < 1 || S_max < 0) return PPD_ERR_INVALID_ARG;
    if (!typical_params_ok(temperature, epsilon, delta)) return PPD_ERR_INVALID_ARG;
    if ((double)B * T * V > 9.0e15) return PPD_ERR_INVALID_ARG;
    AcceptArgs a{cand_tokens, parent, prefix_len, accept_len, path, next_token, new_prefix_len,
                 dev_status, T, V, S_max};
    return cuda_status(ppd::launch_typical_accept(logits, lse, entropy, argmax, a, B, temperature,
                                                  epsilon, delta, static_cast<cudaStream_t>(stream)));
}

// topk [B][n_states][K] int32, kstate [B] int32, then the chain rows'
// log-sum-exps fp32 [B][n_states][kNextMaxEpt].
static size_t next_lse_offset(int B, int n_states, int K)
{
    return align_up(align_up((size_t)B * n_states * K * sizeof(int32_t)) + (size_t)B * sizeof(int32_t));
}

size_t ppd_next_tree_workspace_bytes(int B, int n_states, int K)
{
    if (B < 1 || n_states < 1 || K < 1) return 0;
    return next_lse_offset(B, n_states, K) + align_up((size_t)B * n_states * ppd::kNextMaxEpt * sizeof(float));
}

ppd_status ppd_next_tree_ept(const float *logits, const int32_t *parent,
                             const int32_t *cand_tokens, const int32_t *path,
                             const int32_t *accept_len, const int32_t *next_token, int B, int T,
                             int V, int n_states, int T_next, const int32_t *tmpl_parent,
                             const int32_t *tmpl_rank, int K, int n_ept, int ept_mean,
                             int32_t *next_parent, int32_t *next_cand, int32_t *next_state,
                             int32_t *dev_status, void *workspace, size_t ws_bytes, void *stream)
{
    if (!logits || !parent || !cand_tokens || !path || !accept_len || !next_token || !tmpl_parent ||
        !tmpl_rank || !next_parent || !next_cand || !next_state || !dev_status || !workspace)
        return PPD_ERR_INVALID_ARG;
    if (B < 1 || T < 1 || T > kMaxT || V < 1 || n_states < 1 || n_states > 128 || T_next < 1 ||
        T_next > kMaxT || K < 1 || K > V || n_ept < 1 || ept_mean < 0 || ept_mean > 1)
        return PPD_ERR_INVALID_ARG;
    if (K > ppd::kNextMaxK || n_ept > ppd::kNextMaxEpt) return PPD_ERR_UNSUPPORTED;
    if ((double)B * T * V > 9.0e15) return PPD_ERR_INVALID_ARG;
    if (ws_bytes < ppd_next_tree_workspace_bytes(B, n_states, K) || !aligned(workspace, kAlign))
        return PPD_ERR_INVALID_ARG;
    int32_t *topk = static_cast<int32_t *>(workspace);
    int32_t *kstate = reinterpret_cast<int32_t *>(static_cast<char *>(workspace) +
                                                  align_up((size_t)B * n_states * K * sizeof(int32_t)));
    float *lse = reinterpret_cast<float *>(static_cast<char *>(workspace) + next_lse_offset(B, n_states, K));
    return cuda_status(ppd::launch_next_tree(
        logits, parent, cand_tokens, path, accept_len, next_token, B, T, V, n_states, T_next,
        tmpl_parent, tmpl_rank, K, n_ept, ept_mean, topk, kstate, lse, num_sms(),
        next_parent, next_cand, next_state, dev_status, static_cast<cudaStream_t>(stream)));
}

ppd_status ppd_next_tree(const float *logits, const int32_t *parent, const int32_t *cand_tokens,
                         const int32_t *path, const int32_t *accept_len, const int32_t *next_token,
                         int B, int T, int V, int n_states, int T_next, const int32_t *tmpl_parent,
                         const int32_t *tmpl_rank, int K, int n_ept, int32_t *next_parent,
                         int32_t *next_cand, int32_t *next_state, int32_t *dev_status,
                         void *workspace, size_t ws_bytes, void *stream)
{
    return ppd_next_tree_ept(logits, parent, cand_tokens, path, accept_len, next_token, B, T, V,
                             n_states, T_next, tmpl_parent, tmpl_rank, K, n_ept, 0, next_parent,
                             next_cand, next_state, dev_status, workspace, ws_bytes, stream);
}

ppd_status ppd_selftest_umma(const void *a, const void *b, float *d, int mode, int N, void *stream)
{
    if (!a || !b || !d || mode < 0 || mode > 3 || N < 16 || N > 256 || N % 16 != 0)
        return PPD_ERR_INVALID_ARG;
    if (mode == 3 && N > 128) return PPD_ERR_INVALID_ARG;
    if (mode != 0 && N % 8 != 0) return PPD_ERR_INVALID_ARG;
    if (!aligned(a, 16) || !aligned(b, 16) || !aligned(d, 4)) return PPD_ERR_INVALID_ARG;
    CUtensorMap ma, mb;
    std::memset(&ma, 0, sizeof ma);
    std::memset(&mb, 0, sizeof mb);
    if (mode == 3) {
        // A is written to TMEM by threads, B to shared memory: no tensor maps
    } else if (mode == 0) {
        if (!encode_2d(&ma, a, 128, 128, 128) || !encode_2d(&mb, b, 128, N, N)) return PPD_ERR_CUDA;
    } else {
        if (!encode_2d(&ma, a, mode == 2 ? 64 : 128, 128, 128)) return PPD_ERR_CUDA;
        mb = ma;
    }
    return cuda_status(ppd::launch_selftest_umma(ma, mb, a, b, d, mode, N, static_cast<cudaStream_t>(stream)));
}

// ------------------------------------------------------------------ 4-bit cache, eviction, sampling

// Rows that a slice holds at most: kernels count rows in 32 bits, and steps pass the last one.
constexpr int kMaxRows = 2147483647 - 65536;

// Shapes of a 4-bit cache's slices; G query heads share a K/V head.
static bool kv4_dims_ok(int L, int B, int H, int G, int T, int D, int S_max)
{
    if (L < 1 || B < 1 || H < 1 || G < 1 || T < 1 || S_max < 1 || (D != 64 && D != 128)) return false;
    const double slices = (double)L * B * H;
    return slices * 64 <= 2147483647.0 && slices * G * T <= 2147483647.0 && slices * S_max * D <= 9.0e15;
}

ppd_status ppd_kv4_append(const void *k_new, const void *v_new, uint8_t *k_cache, uint8_t *k_scale,
                          uint8_t *v_cache, uint8_t *v_scale, const int32_t *rows,
                          const int32_t *start, const int32_t *n_new, int L, int B, int H, int T,
                          int D, int S_max, ppd_dtype dt, int32_t *dev_status, void *stream)
{
    if (!k_new || !v_new || !k_cache || !k_scale || !v_cache || !v_scale || !start || !n_new || !dev_status)
        return PPD_ERR_INVALID_ARG;
    if (!kv4_dims_ok(L, B, H, 1, T, D, S_max) || (dt != PPD_BF16 && dt != PPD_F32)) return PPD_ERR_INVALID_ARG;
    if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) ||
        !aligned(k_scale, 16) || !aligned(v_scale, 16))
        return PPD_ERR_INVALID_ARG;
    const size_t cached = (size_t)L * B * H * S_max, fresh = (size_t)L * B * H * T * D * (dt == PPD_F32 ? 4 : 2), nb = (size_t)B * 4;
    if (share_memory({{k_cache, cached * (D / 2)}, {k_scale, cached * (D / 32)}, {v_cache, cached * (D / 2)}, {v_scale, cached * (D / 32)}, {dev_status, nb}},
                     {{k_new, fresh}, {v_new, fresh}, {rows, nb * T}, {start, nb}, {n_new, nb}}))
        return PPD_ERR_INVALID_ARG;
    if (T > 65535 * 64 || S_max > kMaxRows) return PPD_ERR_UNSUPPORTED;
    ppd::Kv4AppendParams p{k_new, v_new, k_cache, v_cache, k_scale, v_scale, rows, start, n_new, dev_status,
                           (long long)L * B * H, B, H, T, D, S_max, dt == PPD_F32};
    return cuda_status(ppd::launch_kv4_append(p, static_cast<cudaStream_t>(stream)));
}

ppd_status ppd_kv4_read(const uint8_t *cache, const uint8_t *scale, const int32_t *start,
                        const int32_t *n, int L, int B, int H, int N, int D, int S_max, void *out,
                        ppd_dtype dt, void *stream)
{
    if (!cache || !scale || !start || !n || !out) return PPD_ERR_INVALID_ARG;
    if (!kv4_dims_ok(L, B, H, 1, N, D, S_max) || (dt != PPD_BF16 && dt != PPD_F32)) return PPD_ERR_INVALID_ARG;
    if (!aligned(cache, 16) || !aligned(scale, 16) || !aligned(out, 16)) return PPD_ERR_INVALID_ARG;
    const size_t cached = (size_t)L * B * H * S_max, nb = (size_t)B * 4;
    if (share_memory({{out, (size_t)L * B * H * N * D * (dt == PPD_F32 ? 4 : 2)}},
                     {{cache, cached * (D / 2)}, {scale, cached * (D / 32)}, {start, nb}, {n, nb}}))
        return PPD_ERR_INVALID_ARG;
    if (S_max > kMaxRows) return PPD_ERR_UNSUPPORTED;
    ppd::Kv4ReadParams p{cache, scale, start, n, out, (long long)L * B * H, B, H, N, D, S_max, dt == PPD_F32};
    return cuda_status(ppd::launch_kv4_read(p, static_cast<cudaStream_t>(stream)));
}

// Parts that the keys of a slice are shared out to, blocks of which `per_sm` fit an SM: the number
// with the shortest time of all waves of blocks, a part counting as its chunks of 32 keys and
// eight more for a block's start and end (960 slices of 1024 keys: 47 us, and 58 us with none
// for them; 32 slices of 10,000 keys: 20 us, and 82 us as whole slices).  A part has at least
// eight chunks, two a warp.
static int kv4_splits(long long slices, int T, int S_max, int per_sm)
{
    const long long slots = (long long)per_sm * num_sms();
    const long long chunks = (S_max + 31) / 32 + (T + 31) / 32;
    long long best = -1, most = chunks / 8;
    int splits = 1;
    if (most > 8 * slots / slices) most = 8 * slots / slices;
    for (long long n = 1; n <= most || n == 1; ++n) {
        const long long cost = (slices * n + slots - 1) / slots * ((chunks + n - 1) / n + 8);
        if (best < 0 || cost < best) best = cost, splits = (int)n;
    }
    return splits;
}

// How an attention call runs: few query rows of a slice in registers, its keys in `splits`
// parts; more on the tensor cores in blocks of tp rows, all key tiles shared out (`share`; a batch
// that the sharing's plan holds).  Registers / tensor cores, 2048 keys, 64 x 32 slices and 32:
//   8 rows, D = 128    170 / 250 us    13 / 15 us
//   12 rows            235 / 250 us    21 / 15 us   (two blocks of eight; of short contexts the latter alike)
//   16 rows, D = 64     79 /  97 us    (64 x 16 slices)
// Blocks of 32 rows against 64 where 32 hold them all: 128 and 145 us (32 x 32 slices).
struct Kv4Ws {
    size_t o, ml, rec, total;
    int row_blocks, splits, tp, share;
};
static Kv4Ws kv4_workspace(int L, int B, int H, int G, int T, int D, int S_max)
{
    Kv4Ws w{};
    const long long slices = (long long)L * B * H, rows = (long long)G * T;
    w.splits = 1;
    if (rows > (D == 64 ? 16 : 8)) {
        w.tp = rows <= 32 ? 32 : 64;
        w.row_blocks = (int)((rows + w.tp - 1) / w.tp);
        // whole units where sharing their tiles out would save less than it costs (about six tiles'
        // time: the merge grid and the parts' way through memory).  Whole / shared, 64 tokens: 23 / 20 us
        // (8 slices of 2048 keys), 29 / 40 us (256 of 1024)
        const long long units = slices * w.row_blocks, t_u = (S_max + 127) / 128 + (T + 127) / 128, sms = split_grid();
        w.share = B <= ppd::kSplitMaxB && units * t_u <= 2147483647 && (units * t_u + sms - 1) / sms + 6 < (units + sms - 1) / sms * t_u;
        if (w.share) {
            w.rec = align_up((size_t)2 * split_grid() * ppd::kv4_slot_floats(D, w.tp) * 4);
            w.total = align_up(w.rec + (size_t)split_grid() * sizeof(ppd::SplitRecord));
        }
        return w;
    }
    w.splits = kv4_splits(slices, T, S_max, rows <= 8 ? 4 : 3);
    if (w.splits > 1) {
        const size_t n = (size_t)slices * w.splits * rows;
        w.ml = align_up(n * D * 4);
        w.total = align_up(w.ml + n * 8);
    }
    return w;
}

size_t ppd_kv4_attention_workspace_bytes(int L, int B, int H, int G, int T, int D, int S_max)
{
    if (!kv4_dims_ok(L, B, H, G, T, D, S_max) || T > kMaxT || S_max > kMaxRows) return 0;
    return kv4_workspace(L, B, H, G, T, D, S_max).total;
}

ppd_status ppd_tree_attention_kv4(const void *q, const uint8_t *k_cache, const uint8_t *k_scale,
                                  const uint8_t *v_cache, const uint8_t *v_scale, const void *k_tree,
                                  const void *v_tree, const int32_t *prefix_len, const int32_t *parent,
                                  int L, int B, int H, int G, int T, int D, int S_max, ppd_dtype dt,
                                  float scale, void *out, float *lse, int32_t *dev_status,
                                  void *workspace, size_t ws_bytes, void *stream)
{
    if (!q || !k_cache || !k_scale || !v_cache || !v_scale || !k_tree || !v_tree || !prefix_len || !parent ||
        !out || !dev_status)
        return PPD_ERR_INVALID_ARG;
    if (!kv4_dims_ok(L, B, H, G, T, D, S_max) || T > kMaxT || (dt != PPD_BF16 && dt != PPD_F32) || !std::isfinite(scale))
        return PPD_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(k_scale, 16) || !aligned(v_cache, 16) ||
        !aligned(v_scale, 16) || !aligned(k_tree, 16) || !aligned(v_tree, 16) || !aligned(out, 16) || !aligned(lse, 4))
        return PPD_ERR_INVALID_ARG;
    if (S_max > kMaxRows) return PPD_ERR_UNSUPPORTED;
    const long long slices = (long long)L * B * H;
    const Kv4Ws w = kv4_workspace(L, B, H, G, T, D, S_max);
    const bool ws_ok = workspace && ws_bytes >= w.total && aligned(workspace, kAlign);
    const size_t cached = (size_t)slices * S_max, rows = (size_t)slices * G * T, nb = (size_t)B * 4, elem = dt == PPD_F32 ? 4 : 2;
    const Mem scratch{ws_ok && w.total ? workspace : nullptr, w.total}, o{out, rows * D * 2}, l{lse, rows * 4}, st{dev_status, nb}, q_rows{q, rows * D * elem};
    if (share_memory({o, l, st, scratch},
                     {{k_cache, cached * (D / 2)}, {k_scale, cached * (D / 32)}, {v_cache, cached * (D / 2)}, {v_scale, cached * (D / 32)},
                      {k_tree, (size_t)slices * T * D * elem}, {v_tree, (size_t)slices * T * D * elem}, {prefix_len, nb}, {parent, nb * T}}) ||
        share_memory({l, st, scratch}, {q_rows}) || (!(q == out && dt == PPD_BF16) && share_memory({o}, {q_rows})))
        return PPD_ERR_INVALID_ARG;
    ppd::Kv4AttnParams p{};
    p.q = q;
    p.k_cache = k_cache, p.k_scale = k_scale, p.v_cache = v_cache, p.v_scale = v_scale;
    p.k_tree = k_tree, p.v_tree = v_tree;
    p.prefix_len = prefix_len, p.parent = parent;
    p.out = static_cast<uint16_t *>(out);
    p.lse = lse;
    p.dev_status = dev_status;
    p.scale_bytes = (size_t)slices * S_max * (D / 32);
    p.slices = slices;
    p.B = B, p.H = H, p.G = G, p.T = T, p.S_max = S_max, p.f32 = dt == PPD_F32;
    p.scale_log2 = (scale > 0.f ? scale : 1.0f / std::sqrt((float)D)) * 1.4426950408889634f;
    if (w.tp) {
        ppd::AttnParams a{};
        a.prefix_len = prefix_len, a.parent = parent;
        a.dev_status = dev_status;
        a.L = L, a.B = B, a.H = H, a.T = T, a.S_max = S_max;
        if (slices * w.row_blocks > 2147483647ll) return PPD_ERR_UNSUPPORTED;
        a.n_qb = w.row_blocks;
        a.n_units = (int)(slices * w.row_blocks);
        a.n_tt = (T + 127) / 128;
        a.cluster = 1;
        a.scale_log2 = p.scale_log2;
        const long long tiles = (long long)a.n_units * ((S_max + 127) / 128 + a.n_tt);
        a.split = w.share && ws_ok;
        if (a.split) {
            a.split_part = static_cast<float *>(workspace);
            a.split_rec = reinterpret_cast<ppd::SplitRecord *>(static_cast<uint8_t *>(workspace) + w.rec);
        }
        const long long most = a.split ? tiles : a.n_units;
        const int grid = (int)(most < split_grid() ? most : split_grid());
        return cuda_status(ppd::launch_kv4_attention_wide(a, p, D, w.tp, grid, static_cast<cudaStream_t>(stream)));
    }
    p.splits = ws_ok ? w.splits : 1;
    if (p.splits > 1) {
        p.part_o = static_cast<float *>(workspace);
        p.part_ml = reinterpret_cast<float2 *>(static_cast<uint8_t *>(workspace) + w.ml);
    }
    if (slices * p.splits > 2147483647ll) return PPD_ERR_UNSUPPORTED;
    return cuda_status(ppd::launch_kv4_attention(p, D, static_cast<cudaStream_t>(stream)));
}

ppd_status ppd_kv_weight_add(const void *q, const float *lse, const void *k_cache, const uint8_t *k_scale,
                             const void *k_tree, const int32_t *path, const int32_t *accept_len,
                             const int32_t *prefix_len, int L, int B, int H, int G, int T, int D, int S_max,
                             ppd_dtype dt, float scale, float *weight, void *stream)
{
    if (!q || !lse || !k_cache || !k_tree || !path || !accept_len || !prefix_len || !weight) return PPD_ERR_INVALID_ARG;
    if (!kv4_dims_ok(L, B, H, G, T, D, S_max) || T > kMaxT || (dt != PPD_BF16 && dt != PPD_F32) || !std::isfinite(scale))
        return PPD_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(k_scale, 16) || !aligned(k_tree, 16) || !aligned(lse, 4) ||
        !aligned(weight, 4))
        return PPD_ERR_INVALID_ARG;
    const size_t slices = (size_t)L * B * H, rows = slices * G * T, cached = slices * S_max, nb = (size_t)B * 4, elem = dt == PPD_F32 ? 4 : 2;
    if (share_memory({{weight, cached * 4}},
                     {{q, rows * D * elem}, {lse, rows * 4}, {k_cache, cached * (k_scale ? D / 2 : 2 * D)}, {k_scale, cached * (D / 32)},
                      {k_tree, slices * T * D * elem}, {path, nb * T}, {accept_len, nb}, {prefix_len, nb}}))
        return PPD_ERR_INVALID_ARG;
    if (S_max > kMaxRows) return PPD_ERR_UNSUPPORTED;
    ppd::KvWeightParams p{};
    p.q = q;
    p.lse = lse;
    p.k_cache = static_cast<const uint8_t *>(k_cache);
    p.k_scale = k_scale;
    p.k_tree = k_tree;
    p.path = path, p.accept_len = accept_len, p.prefix_len = prefix_len;
    p.weight = weight;
    p.slices = (long long)L * B * H;
    p.B = B, p.H = H, p.G = G, p.T = T, p.S_max = S_max, p.f32 = dt == PPD_F32;
    p.scale_log2 = (scale > 0.f ? scale : 1.0f / std::sqrt((float)D)) * 1.4426950408889634f;
    p.scale_bytes = (size_t)p.slices * S_max * (D / 32);
    p.splits = kv4_splits(p.slices, T, S_max, ppd::kv_weight_blocks(k_scale != nullptr));
    return cuda_status(ppd::launch_kv_weight(p, D, static_cast<cudaStream_t>(stream)));
}

ppd_status ppd_kv_evict(const float *weight, float *out_weight, const void *const *planes, void *const *out_planes,
                        const int *row_bytes, int n_planes, const int32_t *length, int L, int B, int H, int S_max,
                        int S_out, int budget, int n_sink, int n_recent, int32_t *kept, int32_t *new_len,
                        int32_t *dev_status, void *stream)
{
    if (!weight || !out_weight || !length || !kept || !new_len || !dev_status || n_planes < 0 ||
        n_planes >= ppd::kMaxPlanes || (n_planes > 0 && (!planes || !out_planes || !row_bytes)))
        return PPD_ERR_INVALID_ARG;
    const double slices = (double)L * B * H;
    if (L < 1 || B < 1 || H < 1 || S_max < 1 || S_out < 1 || slices * 64 > 2147483647.0) return PPD_ERR_INVALID_ARG;
    if (budget < 1 || budget > S_max || budget > S_out || n_sink < 0 || n_recent < 0 || n_sink > budget ||
        n_recent > budget - n_sink)
        return PPD_ERR_INVALID_ARG;
    if (!aligned(weight, 4) || !aligned(out_weight, 4) || slices * S_max * 1024 > 9.0e15 || slices * S_out * 1024 > 9.0e15)
        return PPD_ERR_INVALID_ARG;
    // every block reads the lengths: none may be written meanwhile
    const size_t nb = (size_t)B * 4;
    const Mem kept_m{kept, (size_t)slices * budget * 4}, new_len_m{new_len, nb}, status_m{dev_status, nb}, length_m{length, nb};
    if (share_memory({kept_m, new_len_m, status_m}, {length_m})) return PPD_ERR_INVALID_ARG;
    if (S_max > kMaxRows || S_out > kMaxRows) return PPD_ERR_UNSUPPORTED;
    ppd::KvEvictParams p{};
    p.weight = weight;
    p.length = length;
    p.kept = kept;
    p.new_len = new_len;
    p.dev_status = dev_status;
    p.slices = (long long)L * B * H;
    p.B = B, p.H = H, p.S_max = S_max, p.S_out = S_out, p.budget = budget, p.sink = n_sink, p.recent = n_recent;
    p.planes = n_planes + 1;
    for (int i = 0; i <= n_planes; ++i) {
        ppd::KvPlane &pl = p.plane[i];
        pl.src = i < n_planes ? planes[i] : weight;
        pl.dst = i < n_planes ? out_planes[i] : out_weight;
        pl.row_bytes = i < n_planes ? row_bytes[i] : 4;
        if (!pl.src || !pl.dst || pl.row_bytes < 1 || pl.row_bytes > 1024) return PPD_ERR_INVALID_ARG;
        if (pl.src == pl.dst && S_out != S_max) return PPD_ERR_INVALID_ARG;
        pl.unit = 16;
        while (pl.row_bytes % pl.unit || !aligned(pl.src, pl.unit) || !aligned(pl.dst, pl.unit)) pl.unit /= 2;
    }
    // a destination may be its own source, and shares no byte with another plane; the other outputs
    // share none with a plane
    for (int i = 0; i < p.planes; ++i) {
        const Mem src{p.plane[i].src, (size_t)p.slices * S_max * p.plane[i].row_bytes}, dst{p.plane[i].dst, (size_t)p.slices * S_out * p.plane[i].row_bytes};
        if (share_memory({dst}, {length_m}) || share_memory({kept_m, new_len_m, status_m}, {src, dst})) return PPD_ERR_INVALID_ARG;
        for (int j = 0; j < p.planes; ++j) {
            const size_t ni = (size_t)p.slices * S_out * p.plane[i].row_bytes;
            const size_t ns = (size_t)p.slices * S_max * p.plane[j].row_bytes;
            const size_t nd = (size_t)p.slices * S_out * p.plane[j].row_bytes;
            if (i != j && overlaps(p.plane[i].dst, ni, p.plane[j].dst, nd)) return PPD_ERR_INVALID_ARG;
            if (!(i == j && p.plane[i].src == p.plane[i].dst) && overlaps(p.plane[i].dst, ni, p.plane[j].src, ns))
                return PPD_ERR_INVALID_ARG;
        }
    }
    for (int i = 0; i < p.planes; ++i) {
        ppd::KvPlane &pl = p.plane[i];
        const int per_row = pl.row_bytes / pl.unit;
        if (pl.src == pl.dst) {
            // in place: columns of 32 bytes or more, until the blocks fill the GPU twice
            const int most = pl.row_bytes / 32;
            pl.parts = 1;
            while (pl.parts * 2 <= most && per_row % (pl.parts * 2) == 0 && p.slices * pl.parts < 4ll * num_sms()) pl.parts *= 2;
        } else {
            const long long steps = ((long long)budget * per_row + 1023) / 1024;
            pl.parts = (int)((steps + 3) / 4);
        }
        p.move_blocks += pl.parts;
    }
    if ((double)p.slices * p.move_blocks > 2147483647.0) return PPD_ERR_UNSUPPORTED;
    return cuda_status(ppd::launch_kv_evict(p, static_cast<cudaStream_t>(stream)));
}

ppd_status ppd_sample_accept(const float *logits, const int32_t *cand_tokens, const int32_t *parent,
                             const int32_t *prefix_len, const float *draft_probs, const int32_t *draft_row,
                             const float *u, const float *noise, int B, int T, int V, int n_draft, int S_max,
                             float temperature, int32_t *accept_len, int32_t *path, int32_t *next_token,
                             int32_t *new_prefix_len, float *accept_prob, int32_t *dev_status, void *stream)
{
    if (!logits || !cand_tokens || !parent || !prefix_len || !u || !noise || !accept_len || !path || !next_token ||
        !new_prefix_len || !dev_status || !draft_probs != !draft_row)
        return PPD_ERR_INVALID_ARG;
    if (B < 1 || T < 1 || T > kMaxT || V < 1 || S_max < 1 || (draft_probs && n_draft < 1) || (double)B * T * V > 9.0e15 ||
        (double)B * 8 > 2147483647.0 || (draft_probs && (double)B * n_draft * V > 9.0e15))
        return PPD_ERR_INVALID_ARG;
    if (!std::isfinite(temperature) || temperature <= 0.f || !std::isfinite(1.4426950408889634f / temperature))
        return PPD_ERR_INVALID_ARG;
    if (!aligned(logits, 4) || !aligned(draft_probs, 4) || !aligned(u, 4) || !aligned(noise, 4) || !aligned(accept_prob, 4))
        return PPD_ERR_INVALID_ARG;
    // as many CTAs a sequence as the GPU holds for all of them at once (three an SM, by threads and
    // by a share of up to 50 KB), and none for less than four elements a thread: a small
    // vocabulary's passes are their barriers (80 sequences of 1024 tokens: 24 us with four CTAs each)
    int cluster = ppd::kMaxCluster;
    auto share = [&](int c) { return ((V + c - 1) / c + 3) & ~3; };
    while (cluster > 1 && (((long long)B * cluster > 3ll * num_sms() && share(cluster / 2) <= 12800) || share(cluster) < 2048)) cluster /= 2;
    const int chunk = share(cluster);
    if (chunk > ppd::kSampleMaxChunk) return PPD_ERR_UNSUPPORTED;
    // the CTAs of a sequence read its entries before one of them writes there, those of another may not have
    const size_t nb = (size_t)B * 4, nodes = nb * T;
    const Mem outs[] = {{accept_len, nb}, {next_token, nb}, {new_prefix_len, nb}, {dev_status, nb}, {path, nodes}, {accept_prob, nodes}};
    const Mem ins[] = {{prefix_len, nb}, {cand_tokens, nodes}, {parent, nodes}, {draft_row, nodes}, {u, nodes}};
    for (const Mem &o : outs) {
        if (share_memory({o}, {{logits, nodes * V}, {noise, nb * V}, {draft_probs, nb * V * (draft_probs ? n_draft : 0)}})) return PPD_ERR_INVALID_ARG;
        for (const Mem &i : ins)
            if (!(o.p == i.p && o.n == i.n) && share_memory({o}, {i})) return PPD_ERR_INVALID_ARG;
    }
    if (share_memory({outs[0], outs[1], outs[2], outs[3], outs[4], outs[5]}, {})) return PPD_ERR_INVALID_ARG;
    ppd::SampleParams p{logits, cand_tokens, parent, prefix_len, draft_probs, draft_row, u, noise, accept_len, path,
                        next_token, new_prefix_len, dev_status, accept_prob, B, T, V, S_max, draft_probs ? n_draft : 0,
                        1.4426950408889634f / temperature, chunk};
    return cuda_status(ppd::launch_sample_accept(p, cluster, static_cast<cudaStream_t>(stream)));
}

// ------------------------------------------------------------------ a pool of pages

// log2 of a page's rows, or -1 where such pages are not supported: powers of two from 8 (a box of
// the attention's copies starts on eight rows) to 256.
static int page_shift(int page)
{
    for (int s = 3; s <= 8; ++s)
        if (page == 1 << s) return s;
    return -1;
}

static bool pool_dims_ok(int L, int H, int D, int page, int n_pages)
{
    if (L < 1 || H < 1 || (D != 64 && D != 128) || page < 1 || n_pages < 1) return false;
    return (double)n_pages * page <= (double)kMaxRows && (double)L * n_pages * H < 2147483647.0;
}

ppd_status ppd_page_assign(const int32_t *old_len, const int32_t *new_len, int B, int page, int n_pages, int max_pages,
                           int max_slots, int32_t *table, int32_t *free_pages, const int32_t *n_free, int32_t *new_n_free,
                           int32_t *out_len, int32_t *slots, int32_t *slot_start, int32_t *dev_status, void *stream)
{
    if (!old_len || !new_len || !table || !free_pages || !n_free || !new_n_free || !out_len || !slots || !slot_start || !dev_status)
        return PPD_ERR_INVALID_ARG;
    if (B < 1 || page < 1 || n_pages < 1 || max_pages < 1 || max_slots < 1) return PPD_ERR_INVALID_ARG;
    const size_t nb = (size_t)B * 4;
    if (share_memory({{table, nb * max_pages}, {free_pages, (size_t)n_pages * 4}, {new_n_free, 4}, {out_len, nb}, {slots, (size_t)max_slots * 4},
                      {slot_start, nb + 4}, {dev_status, nb}},
                     {{old_len, nb}, {new_len, nb}, {n_free, 4}}))
        return PPD_ERR_INVALID_ARG;
    if (page_shift(page) < 0 || B > ppd::kMaxAssign || (double)n_pages * page > kMaxRows || (double)max_pages * page > kMaxRows ||
        (double)B * max_pages > 2147483647.0 || max_slots > kMaxRows)
        return PPD_ERR_UNSUPPORTED;
    ppd::PageAssignParams p{old_len, new_len, n_free, table, free_pages, new_n_free, out_len, slots, slot_start, dev_status,
                            B, page_shift(page), n_pages, max_pages, max_slots, aligned(slots, 16)};
    return cuda_status(ppd::launch_page_assign(p, num_sms(), static_cast<cudaStream_t>(stream)));
}

ppd_status ppd_page_append(const void *k_new, const void *v_new, void *k_pages, void *v_pages, const int32_t *rows,
                           const int32_t *slots, const int32_t *slot_start, int L, int B, int H, int T, int D, int page,
                           int n_pages, int max_slots, ppd_dtype dt, int32_t *dev_status, void *stream)
{
    if (!k_new || !v_new || !k_pages || !v_pages || !slots || !slot_start || !dev_status) return PPD_ERR_INVALID_ARG;
    if (B < 1 || T < 1 || max_slots < 1 || (dt != PPD_BF16 && dt != PPD_F32) || !pool_dims_ok(L, H, D, page, n_pages))
        return PPD_ERR_INVALID_ARG;
    if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16)) return PPD_ERR_INVALID_ARG;
    const double slices = (double)L * B * H;
    if (slices * T * D > 9.0e15) return PPD_ERR_INVALID_ARG;
    const size_t pool = (size_t)L * n_pages * H * page * D * 2, fresh = (size_t)L * B * H * T * D * (dt == PPD_F32 ? 4 : 2), nb = (size_t)B * 4;
    if (share_memory({{k_pages, pool}, {v_pages, pool}, {dev_status, nb}},
                     {{k_new, fresh}, {v_new, fresh}, {rows, nb * T}, {slots, (size_t)max_slots * 4}, {slot_start, nb + 4}}))
        return PPD_ERR_INVALID_ARG;
    if (page_shift(page) < 0 || slices * ppd::page_append_chunks(T) > 2147483647.0) return PPD_ERR_UNSUPPORTED;
    ppd::PageAppendParams p{k_new, v_new, k_pages, v_pages, slots, slot_start, rows, dev_status, (long long)L * B * H, B, H, T, D, n_pages,
                            page_shift(page), max_slots, dt == PPD_F32, 0};
    return cuda_status(ppd::launch_page_append(p, static_cast<cudaStream_t>(stream)));
}

// How an attention call over pages runs: units of query rows of a slice (n_qb of them), how they are
// shared out, and where the bf16 copies of fp32 operands and the work split's states lie in the
// workspace.
struct PagedWs {
    int rows, n_qb, n_tt, pair_units;
    AttnPlan plan;
    size_t rec, part, total;
};

// Slices of more than 64 rows, by the time that each way takes, in microseconds a job of t_u tiles and at
// its ends (the tables' capacity standing in for the lengths), as measured with D = 128, pages of
// 32: a tile of 128 queries 1.09, or 1.47 where every SM streams keys of its own, of a pair of blocks
// 2.05; whole jobs' ends 6, a cluster's 12, and the work split's 24 (two jobs a CTA, 130 KB of
// partial state each, and the merge).  Whole / clusters / shared out, heads of 64 tokens:
//   16 slices, 4 heads, 3001 rows    30.5 /  18.9 /  30.0     96 of 4, ragged to 5001   82.2 /      /  64.3
//   8 of 4, 20,001                    149 /  37.3 /  43.2     64 of 4                   46.2 /      /  52.1
//   40 of 2, 4001                    37.5 /  21.3 /  27.6     80 of 4                   82.5 /      /  58.0
// (units of the work split: pairs of blocks; single ones took 5, 10 and 20 us longer on 96 slices of 4 heads,
// 64 and 80 of 8).
static void plan_paged_rows(PagedWs &w, long long slices, long long t_u, int B, bool workspace)
{
    const long long sms = split_grid(), blocks = (w.rows + 127) / 128, pairs = (blocks + 1) / 2;
    auto rounds = [&](long long jobs) { return (double)((jobs + sms - 1) / sms); };
    const double alone = slices * blocks >= sms ? 1.47 : 1.09;
    double best = rounds(slices * blocks) * alone * t_u + 6;
    if (blocks > 1) best = std::min(best, rounds(slices * pairs) * 2.05 * t_u + 6);
    w.plan = {0, 1};
    w.n_qb = (int)blocks;
    w.pair_units = 0;
    for (int c = 2; c <= ppd::kMaxCluster && c <= t_u && slices * blocks * c <= sms; ++c) {
        const double cost = 1.09 * ((t_u + c - 1) / c) + 12;
        if (cost < best && slices * blocks <= ppd::max_attention_clusters(c)) {
            best = cost;
            w.plan.cluster = c;
        }
    }
    const double shared = rounds(slices * pairs * t_u) * (blocks > 1 ? 2.05 : 1.47) + 24;
    // (a twentieth less: lengths are seldom alike, and whole jobs take the longest first)
    if (workspace && B <= ppd::kSplitMaxB && slices * pairs * t_u <= 2147483647ll && shared < 0.95 * best) {
        w.plan = {1, 1};
        if (blocks > 1) {
            w.pair_units = 1;
            w.n_qb = (int)pairs;
        }
    }
}

// Slices of up to 64 rows, fewer than SMs, by the time that each way takes, in microseconds (D = 128,
// pages of 16, the tables' capacity standing in for the lengths): a tile 0.62 and more the more SMs stream; ends
// 6.2, of the work split 12.5 and 0.8 for each round of the merge's loads past one and a half.  Lengths
// of several requests are taken to average 0.8 of the longest.  Clusters / shared out (4 query rows):
//   2 slices of 6000 rows   10.4 / 13.3    8 of 6000     12 / 15.9       32 of 6000    17.0 / 20.4
//   2 of 10,000             12.9 / 17.0    8 of 16,000   19.5 / 19.5     32 of 20,000  47.6 / 46.0
//   2 of 16,000             17.0 / 16.6    8 of 64,000   64.2 / 47.2     56 of 6000    28.4 / 27.6
//   2 of 64,000             55.0 / 23.2    16 of 6000    13.3 / 17.0     96 of 6000 (whole)  48.5 / 42.9
static AttnPlan plan_paged_key(long long slices, long long t_u, int B, int rows, int D, bool may_split)
{
    const long long sms = split_grid();
    auto tile = [](long long ctas) { return 0.62 + 0.0045 * (double)ctas; };
    AttnPlan plan{0, 1};
    double best = tile(slices) * (double)t_u + 6.2;
    for (int c = 2; c <= ppd::kMaxCluster && c <= t_u && slices * c <= sms; ++c) {
        const double cost = tile(slices * c) * (double)((t_u + c - 1) / c) + 6.2;
        if (cost < best && slices <= ppd::max_attention_clusters(c)) {
            best = cost;
            plan.cluster = c;
        }
    }
    const int ways = ppd::paged_merge_ways(ppd::paged_merge_threads(rows, slices, (int)sms), rows, D);
    const double trips = (double)sms / (double)slices / 4 / ways;   // of the merge's loads
    const double shared = 1.35 * (B > 1 ? 0.8 : 1.0) * (double)((slices * t_u + sms - 1) / sms) + 12.5 + 0.8 * std::max(0.0, trips - 1.5);
    if (may_split && shared < best) plan = {1, 1};
    return plan;
}

static PagedWs paged_workspace(int L, int B, int H, int G, int T, int D, int S_max, ppd_dtype dt, bool workspace)
{
    PagedWs w{};
    const long long slices = (long long)L * B * H, sms = split_grid();
    w.rows = G * T;
    w.n_tt = w.rows > 64 ? (T + 127) / 128 : 1;
    const long long t_u = (S_max + 127) / 128 + w.n_tt;
    if (w.rows > 64) {
        plan_paged_rows(w, slices, t_u, B, workspace);
    } else {
        w.n_qb = 1;
        const bool may_split = workspace && B <= ppd::kSplitMaxB && slices * t_u <= 2147483647ll;
        w.plan = slices < sms ? plan_paged_key(slices, t_u, B, w.rows, D, may_split) : AttnPlan{0, 1};
        // (whole units take the longest first; what their last, partial round costs over a share for every SM
        // has to pay for the work split's merge.  160 slices of up to 4000 rows: whole 44.8 us, shared out 42.9;
        // of 2000 25.5 and 27.7)
        if (may_split && slices >= sms && (slices * t_u + sms - 1) / sms + 20 < (slices + sms - 1) / sms * t_u) w.plan = {1, 1};
    }
    size_t off = dt == PPD_F32 ? align_up((size_t)slices * (w.rows + 2 * (size_t)T) * D * 2) : 0;
    if (w.plan.split) {
        w.rec = off;
        off = align_up(off + (size_t)split_grid() * sizeof(ppd::SplitRecord));
        w.part = off;
        off = align_up(off + (size_t)2 * split_grid() * (w.pair_units ? 2 : 1) * ppd::kSplitRows * (D + 2) * sizeof(float));
    }
    w.total = off;
    return w;
}

static bool paged_dims_ok(int L, int B, int H, int G, int T, int D, int S_max, ppd_dtype dt)
{
    if (!kv4_dims_ok(L, B, H, G, T, D, S_max) || T > kMaxT || (dt != PPD_BF16 && dt != PPD_F32)) return false;
    return (double)G * T <= 1 << 20;
}

size_t ppd_paged_attention_workspace_bytes(int L, int B, int H, int G, int T, int D, int S_max, ppd_dtype dt)
{
    if (!paged_dims_ok(L, B, H, G, T, D, S_max, dt) || S_max > kMaxRows) return 0;
    return paged_workspace(L, B, H, G, T, D, S_max, dt, true).total;
}

ppd_status ppd_tree_attention_paged(const void *q, const void *k_pages, const void *v_pages, const int32_t *table,
                                    const void *k_tree, const void *v_tree, const int32_t *prefix_len,
                                    const int32_t *parent, int L, int B, int H, int G, int T, int D, int page, int n_pages,
                                    int max_pages, ppd_dtype dt, float scale, void *out, float *lse, int32_t *dev_status,
                                    void *workspace, size_t ws_bytes, void *stream)
{
    if (!q || !k_pages || !v_pages || !table || !k_tree || !v_tree || !prefix_len || !parent || !out || !dev_status)
        return PPD_ERR_INVALID_ARG;
    if (max_pages < 1 || !pool_dims_ok(L, H, D, page, n_pages) || !std::isfinite(scale)) return PPD_ERR_INVALID_ARG;
    if ((double)max_pages * page > kMaxRows || page_shift(page) < 0) return PPD_ERR_UNSUPPORTED;
    const int S_max = max_pages * page;
    if (!paged_dims_ok(L, B, H, G, T, D, S_max, dt)) return PPD_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(k_tree, 16) || !aligned(v_tree, 16) ||
        !aligned(out, 16) || !aligned(lse, 4))
        return PPD_ERR_INVALID_ARG;
    PagedWs w = paged_workspace(L, B, H, G, T, D, S_max, dt, true);
    bool ws_ok = workspace && ws_bytes >= w.total && aligned(workspace, kAlign);
    if (dt == PPD_F32 && !ws_ok) return PPD_ERR_INVALID_ARG;
    if (!ws_ok) w = paged_workspace(L, B, H, G, T, D, S_max, dt, false);
    const size_t slices = (size_t)L * B * H, rows = slices * w.rows, tree = slices * T * D * (dt == PPD_F32 ? 4 : 2), nb = (size_t)B * 4;
    const size_t pool = (size_t)L * n_pages * H * page * D * 2;
    if (share_memory({{out, rows * D * 2}, {lse, rows * 4}, {dev_status, nb}, {ws_ok && w.total ? workspace : nullptr, w.total}},
                     {{q, rows * D * (dt == PPD_F32 ? 4 : 2)}, {k_pages, pool}, {v_pages, pool}, {table, nb * max_pages}, {k_tree, tree},
                      {v_tree, tree}, {prefix_len, nb}, {parent, nb * T}}))
        return PPD_ERR_INVALID_ARG;
    if ((double)slices * w.n_qb > 2147483647.0) return PPD_ERR_UNSUPPORTED;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    if (dt == PPD_F32) {
        uint16_t *bq = reinterpret_cast<uint16_t *>(ws), *bk = bq + rows * D, *bv = bk + slices * T * D;
        ppd::RoundArgs r{};
        r.t[0] = {static_cast<const float *>(q), bq, w.rows, 0};
        r.t[1] = {static_cast<const float *>(k_tree), bk, T, 0};
        r.t[2] = {static_cast<const float *>(v_tree), bv, T, 0};
        r.n = 3, r.B = B, r.H = H, r.D = D, r.prefix_len = prefix_len;
        const cudaError_t e = ppd::launch_round_bf16(r, (int64_t)slices, true, s);
        if (e != cudaSuccess) return cuda_status(e);
        q = bq, k_tree = bk, v_tree = bv;
    }
    const int T_pad = (w.rows + 31) & ~31, shift = page_shift(page);
    const uint32_t tree_box = T_pad > 64 ? 128u : (uint32_t)ppd::tree_box_rows(T);
    AttnMaps m;
    if (!encode_3d(&m.q, q, D, w.rows, slices, T_pad > 64 ? 128u : (uint32_t)T_pad) ||
        !encode_3d(&m.kc, k_pages, D, page, (uint64_t)L * n_pages * H, page < 128 ? page : 128) ||
        !encode_3d(&m.vc, v_pages, D, page, (uint64_t)L * n_pages * H, page < 128 ? page : 128) ||
        !encode_3d(&m.kt, k_tree, D, T, slices, tree_box) || !encode_3d(&m.vt, v_tree, D, T, slices, tree_box))
        return PPD_ERR_CUDA;
    ppd::PagedParams p{};
    p.prefix_len = prefix_len, p.parent = parent;
    p.out = static_cast<float *>(out);
    p.lse = lse;
    p.dev_status = dev_status;
    p.L = L, p.B = B, p.H = H, p.T = T, p.T_pad = T_pad, p.S_max = S_max;
    p.n_qb = w.n_qb, p.n_tt = w.n_tt;
    p.n_units = (int)(slices * w.n_qb);
    p.scale_log2 = (scale > 0.f ? scale : 1.0f / std::sqrt((float)D)) * 1.4426950408889634f;
    p.table = table;
    p.max_pages = max_pages, p.n_pages = n_pages, p.n_depth = L * n_pages * H;
    p.page_shift = shift, p.box_shift = shift < 7 ? shift : 7;
    p.rows = w.rows;
    p.pair_units = w.pair_units;
    if (!w.pair_units) ppd::plan_rows(p, split_grid());
    p.cluster = w.plan.cluster;
    if (w.plan.split) {
        p.split = 1;
        p.split_rec = reinterpret_cast<ppd::SplitRecord *>(ws + w.rec);
        p.split_part = reinterpret_cast<float *>(ws + w.part);
    }
    p.set_status = 1;
    p.pdl_wait = 1;
    return cuda_status(ppd::launch_paged_attention(m, p, D, split_grid(), s));
}

ppd_status ppd_token_logprobs(const void *logits, const int32_t *tokens, const int32_t *rows, int B, int T, int V, int n, int K,
                              ppd_dtype dt, float temperature, float *logprob, float *entropy, int32_t *rank,
                              int32_t *top_tokens, float *top_logprobs, int32_t *dev_status, void *stream)
{
    if (!logits || !tokens || !logprob || !entropy || !rank || !dev_status || (K > 0 && (!top_tokens || !top_logprobs)))
        return PPD_ERR_INVALID_ARG;
    if (B < 1 || T < 1 || V < 1 || n < 1 || K < 0 || K > V || (!rows && n > T) || (dt != PPD_BF16 && dt != PPD_F32) ||
        (double)B * T * V > 9.0e15)
        return PPD_ERR_INVALID_ARG;
    if (!std::isfinite(temperature) || temperature <= 0.f || !std::isfinite(1.4426950408889634f / temperature))
        return PPD_ERR_INVALID_ARG;
    const size_t eb = dt == PPD_F32 ? 4 : 2, nb = (size_t)B * 4, items = nb * n;
    if (!aligned(logits, eb) || !aligned(logprob, 4) || !aligned(entropy, 4) || !aligned(top_logprobs, 4)) return PPD_ERR_INVALID_ARG;
    const Mem none{nullptr, 0};
    if (share_memory({{logprob, items}, {entropy, items}, {rank, items}, K ? Mem{top_tokens, items * K} : none,
                      K ? Mem{top_logprobs, items * K} : none, {dev_status, nb}},
                     {{logits, (size_t)B * T * V * eb}, {tokens, items}, {rows, items}}))
        return PPD_ERR_INVALID_ARG;
    if (K > ppd::kLogMaxK || (double)B * n * ppd::kMaxCluster > 2147483647.0 || V > kMaxRows) return PPD_ERR_UNSUPPORTED;
    const float k = 1.4426950408889634f / temperature, span = 138.62943611198906f * temperature;
    const ppd::LogScale scale{k, span, span < 1e30f ? 1048576.f / k : 0.f, k < 1.f ? 0.5f : 1.f, k < 1.f ? 2.f * k : k};
    ppd::LogprobParams p{logits, tokens, rows, logprob, entropy, rank, top_tokens, top_logprobs, dev_status, B, T, V, n, K, dt == PPD_BF16, scale, 1};
    return cuda_status(ppd::launch_token_logprobs(p, num_sms(), static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
