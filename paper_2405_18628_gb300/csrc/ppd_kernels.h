// ppd_kernels.h -- internal launch interface between the C-ABI layer
// (ppd_api.cu) and the kernels.  Not part of the public API.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

namespace ppd {

// A bounded device-side wait gives up after this many nanoseconds of %globaltimer.
constexpr uint64_t kWaitLimitNs = 4000000000ull;

// Tensor maps of the attention operands (bf16, 128-byte swizzle, boxes of
// 64 columns): Q [LBH][T][D] (box rows T_pad), cache K/V [LBH][S_max][D] and
// tree K/V [LBH][T][D] (box rows 128).
struct AttnMaps {
    CUtensorMap q, kc, vc, kt, vt;
};

// The fused verification step's side work (see ppd_attention_common.cuh):
// argmax partials (from the preceding grid, or with in_grid computed by the
// side warps themselves), acceptance, and compaction of the CTA's own
// (layer, sequence, head) slices.
struct FusedStep {
    float *part_val;             // [B*T*splits] partial maxima
    int32_t *part_idx;
    int splits;
    // in_grid != 0: no preceding grid; the side warps compute the partial
    // maxima themselves while the other warps stream K/V.  Chunk c of the
    // [B*T][splits] partial grid is computed by CTA c mod grid; a CTA
    // publishes ready[cta] = tag once its chunks are written, where tag =
    // *epoch + 1 read at its start.  CTA 0 waits until every flag equals tag,
    // then sets *epoch = tag and *all_ready = tag; the other CTAs read
    // partials once *all_ready equals their tag.  Every call has a fresh tag,
    // so no flag needs zeroing.
    int in_grid;
    unsigned long long wait_limit_ns;   // the grid-wide wait gives up after this long
    int withhold_cta;            // diagnostics: this CTA never publishes its flag (-1: none)
    int chunk;                   // logits per chunk (multiple of 4 when vec)
    int vec;                     // 16-byte loads of the logits
    float stat_k;                // log2(e) / temperature (typical acceptance)
    unsigned long long *epoch;   // [1]
    unsigned long long *all_ready;   // [1]
    unsigned long long *ready;   // [grid]
    const int32_t *cand_tokens;  // [B,T]
    int32_t *argmax_out;         // [B,T]
    int32_t *accept_len;         // [B]
    int32_t *path;               // [B,T]
    int32_t *next_token;         // [B]
    int32_t *new_prefix_len;     // [B]
    int32_t *status;             // [B]: zeroed by the grid before (the argmax grid, or with
                                 // in_grid a one-block reset), then raised with atomicMax
    uint8_t *k_cache, *v_cache;  // raw cache storage
    const uint8_t *k_tree, *v_tree;
    int row_bytes;               // D * element size
    int V;
    int *scratch;                // [grid][kSideScratchInts] per-CTA scratch of the side warp
    // typical acceptance (typical != 0): partial softmax statistics from the
    // preceding grid, the logits for p(token), and the rule's parameters
    int typical;
    float *part_stats;           // [B*T*splits][3]
    const float *logits;         // [B,T,V]
    float inv_temp, epsilon, delta;
};

// Largest tree (nodes) of the verification step, and the per-warp scratch
// that acceptance needs: parents, then one 32-bit word per 32 nodes of pass bits.
constexpr int kMaxTree = 512;
constexpr int kAcceptScratchInts = kMaxTree + kMaxTree / 32;

// Per-CTA scratch of the fused step's side warp: acceptance scratch, top-1
// tokens, path, and (typical acceptance) each node's log-sum-exp and entropy.
constexpr int kSideScratchInts = kAcceptScratchInts + 4 * kMaxTree + 8;

struct AttnParams {
    const int32_t *prefix_len;  // [B]
    const int32_t *parent;      // [B,T]
    float *out;                 // [L,B,H,T,D]
    float *lse;                 // [L,B,H,T] or null
    int32_t *dev_status;        // [B] or null (main-loop errors; null in the fused step)
    int L, B, H, T, T_pad, S_max, n_units;
    int n_qb;                   // query blocks of 128 per (layer, sequence, head) slice
    int n_tt;                   // tree-key tiles of 128 per slice
    int pairs;                  // query-row kernel: two blocks of queries of a slice are one job
    int pair_grid;              // with an odd n_qb: the CTAs that take the slices' pairs
    float scale_log2;           // softmax scale * log2(e)
    // Work split: split != 0 shares all units out by their key tiles (launches with
    // fewer units than CTAs, B <= kSplitMaxB); units cut by a range
    // boundary leave partial softmax states in split_part, merged afterwards by
    // launch_split_merge from the per-CTA records in split_rec.
    int split;
    float *split_part;          // [2 * grid][kSplitRows * (D + 2)] partial states
    struct SplitRecord *split_rec;   // [grid]
    // Cluster split: cluster > 1 gives every unit a cluster of that many CTAs, each an
    // equal share of its tiles; their partial states are merged through distributed
    // shared memory.
    int cluster;
    int set_status;             // the attention grid writes every sequence's dev_status itself
    int fused;                  // run the end phase below
    FusedStep fs;
    // Launched as a programmatic dependent of the preceding grid (a chain of
    // ppd_tree_attention calls): the setup that reads no input overlaps that
    // grid, then every thread waits for it before reading any input.
    int pdl_wait;
    // Launched as a programmatic dependent of grids whose results it does not read
    // (a step of more than 64 sequences): a spare warp waits for them, so that this
    // grid's completion says that they are complete too.
    int late_wait;
};

// Attention over pages (ppd_paged.cuh): G query heads share a K/V head, `out` is bf16, S_max
// the rows that a sequence's table can name.
struct PagedParams : AttnParams {
    const int32_t *table;       // [B][max_pages]
    int max_pages, n_pages;
    int n_depth;                // L * n_pages * H
    int page_shift, box_shift;  // log2 of a page's rows, and of min(128, those)
    int rows;                   // query rows of a slice: its G heads' T tokens
    int pair_units;             // work split, more than 128 rows: units are pairs of blocks of 128 rows
};

// Rows of a box of the tree's keys or values in the key-row kernel over pages.
inline __host__ __device__ int tree_box_rows(int T) { return (T + 7) & ~7; }

// Threads of a block of the merge over pages, and how many of them share the parts of eight columns of a row.
// (512 for few slices, which have many parts: 29.5 and 33.4 us for one of 64,000 rows, 8 query rows; 96 of 6000
// rows 43.4 and 42.5.)
inline int paged_merge_threads(int rows, long long slices, int grid) { return rows <= 16 && slices * 8 <= grid ? 512 : 256; }
inline int paged_merge_ways(int threads, int rows, int D) { return rows < threads * 8 / D ? threads * 8 / D / rows : 1; }

// Work split limits: batch size (the per-CTA range search holds the batch in
// two warp-wide registers), CTAs, and query rows of a partial state.
constexpr int kSplitMaxB = 64;
constexpr int kSplitMaxGrid = 256;
constexpr int kSplitRows = 128;

// CTAs of a cluster at most (the portable size).
constexpr int kMaxCluster = 8;

// Clusters of `size` attention CTAs (one per SM) the current device can hold at
// once; 0 when it cannot be asked.
int max_attention_clusters(int size);

// A number >= 0 asked for once: kept in `slot` (plus one; 0: not known yet).  An `ask`
// that fails (a negative answer) counts as 0 this time and is asked again the next.
template <class Ask>
inline int asked_once(std::atomic<int> &slot, Ask ask)
{
    const int got = slot.load(std::memory_order_relaxed);
    if (got > 0) return got - 1;
    const int n = ask();
    if (n < 0) return 0;
    slot.store(n + 1, std::memory_order_relaxed);
    return n;
}

// The unit a CTA has to have merged: it holds the unit's first tile and its
// range ends inside the unit (u = -1: none).  off: the unit's tile 0 among
// the launch's tiles; n_shared: their number.
struct SplitRecord {
    long long off, n_shared;
    int u, n_tiles;
};

// Jobs of a launch without a split: its units, or with p.pairs a slice's pairs of
// blocks and, where their number is odd, a single one.
inline long long whole_jobs(const AttnParams &p)
{
    if (!p.pairs) return p.n_units;
    const long long slices = p.n_units / p.n_qb;
    return (p.n_qb + 1) / 2 * slices;
}

// Whether the query-row kernel's whole jobs are pairs of query blocks, and for
// an odd n_qb the split of the CTAs between pairs and single blocks: the choice with
// the shortest longest queue.  A pair counts as 2 n + 4 and a single block next
// to it as n + 4.5 tiles of 128 x 128 with n prefix tiles (S_max standing in for
// the device-side prefix lengths): three tree tiles each, and the end of a job,
// which only a pair's other stream overlaps.  Without pairs every block streams
// its keys itself: 15 % more a tile (L2), but twice the jobs, so it is the
// choice for launches with few slices (16 x 32 calls of 32 slices, 285 tokens
// over 1500 keys: pairs 36.6 us a call, single blocks 30.1).
inline void plan_rows(AttnParams &p, int num_sms)
{
    p.pairs = 0;
    if (p.T_pad <= 64 || p.n_qb < 2) return;
    const long long S = p.n_units / p.n_qb, G = num_sms, n = (p.S_max + 127) / 128;
    const long long single_all = (23 * (2 * n + 9)) * ((p.n_units + G - 1) / G);   // in 1/40 tiles
    long long best = -1;
    int grid = 0;
    if (p.n_qb & 1) {
        const long long pairs = S * (p.n_qb / 2), Gp = G < pairs + S ? G : pairs + S;
        for (long long g = 1; g < Gp; ++g) {
            const long long a = (4 * n + 8) * ((pairs + g - 1) / g), b = (2 * n + 9) * ((S + Gp - g - 1) / (Gp - g));
            const long long t = a > b ? a : b;
            if (best < 0 || t <= best) {
                best = t;
                grid = (int)g;
            }
        }
    } else {
        const long long jobs = S * (p.n_qb / 2);
        best = (4 * n + 8) * ((jobs + G - 1) / G);
    }
    if (best < 0 || 20 * best > single_all) return;
    p.pairs = 1;
    p.pair_grid = grid;
}

// Whether the launch takes whole jobs of several sequences, whose lengths (known
// to the device alone) may differ.
inline bool whole_ragged(const AttnParams &p)
{
    return p.B > 1 && p.B <= kSplitMaxB && !p.split && p.cluster <= 1;
}

// CTAs of an attention launch: one per SM, at most one per job (with the
// work split: at most one per tile, and kSplitMaxGrid).
inline int attention_grid(const AttnParams &p, int num_sms)
{
    long long grid = num_sms;
    if (p.cluster > 1) return p.n_units * p.cluster;
    if (p.split) {
        const long long max_tiles = (long long)p.n_units * ((p.S_max + 127) / 128 + p.n_tt);
        grid = grid < kSplitMaxGrid ? grid : kSplitMaxGrid;
        grid = grid < max_tiles ? grid : max_tiles;
    } else {
        const long long jobs = whole_jobs(p);
        grid = grid < jobs ? grid : jobs;
    }
    return (int)grid;
}

// Merge the partial states of every cut unit of the attention launch just
// enqueued (one CTA per attention CTA, `grid` of them), after it completes.
cudaError_t launch_split_merge(const AttnParams &p, int D, int grid, cudaStream_t stream);

// Batches up to this size run the fused step (one grid, or an argmax grid then
// the attention grid).
constexpr int kFusedMaxB = 64;

// Dispatches on the padded tree size: up to 64 tokens the key-row kernel
// (ppd_attention_key.cuh), 65..512 the query-row kernel (ppd_attention_rows.cuh).
cudaError_t launch_tree_attention(const AttnMaps &m, const AttnParams &p, int D, int num_sms,
                                  bool programmatic, cudaStream_t stream);
cudaError_t launch_tree_attention_rows(const AttnMaps &m, const AttnParams &p, int D, int num_sms,
                                       bool programmatic, cudaStream_t stream);

// The same over pages, on the padded number of a slice's query rows.
cudaError_t launch_paged_attention(const AttnMaps &m, const PagedParams &p, int D, int num_sms, cudaStream_t stream);
cudaError_t launch_paged_attention_rows(const AttnMaps &m, const PagedParams &p, int D, int num_sms, cudaStream_t stream);

// A kernel launch as a programmatic dependent of the stream's previous grid (it
// may start before that grid completes; the kernel waits with pdl_wait()), in
// clusters of `cluster` (1 1 1: none).
template <typename... KArgs, typename... Args>
inline cudaError_t launch_chained(void (*kern)(KArgs...), dim3 grid, dim3 block, dim3 cluster,
                                  cudaStream_t stream, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    if (cluster.x * cluster.y * cluster.z > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = cluster.x;
        attr[1].val.clusterDim.y = cluster.y;
        attr[1].val.clusterDim.z = cluster.z;
        cfg.numAttrs = 2;
    }
    cfg.attrs = attr;
    return cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
}

// The same with dynamic shared memory (allowed first, once per kernel and device).
template <typename Kern>
inline cudaError_t allow_smem(Kern kern, uint32_t bytes, std::atomic<uint64_t> &configured)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? (1ull << dev) : 0ull;
    if (bit && (configured.load(std::memory_order_acquire) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess) configured.fetch_or(bit, std::memory_order_acq_rel);
    return e;
}

template <typename... KArgs, typename... Args>
inline cudaError_t launch_chained_smem(void (*kern)(KArgs...), dim3 grid, dim3 block, dim3 cluster,
                                       uint32_t smem, cudaStream_t stream, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    if (cluster.x * cluster.y * cluster.z > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = cluster.x;
        attr[1].val.clusterDim.y = cluster.y;
        attr[1].val.clusterDim.z = cluster.z;
        cfg.numAttrs = 2;
    }
    cfg.attrs = attr;
    return cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
}

// Splits per node row of the argmax: about 512 blocks over all rows, chunks of
// at least 2048 logits, at most 64 splits.
inline int argmax_split_count(int64_t rows, int V)
{
    if (rows <= 0) return 1;
    int64_t want = (512 + rows - 1) / rows;
    int64_t cap = V / 2048;
    if (cap > 64) cap = 64;
    if (cap < 1) cap = 1;
    if (want > cap) want = cap;
    if (want < 1) want = 1;
    return (int)want;
}

// Node argmax in two steps: per-(row, split) partial maxima, then a combine.
// part_stats (3 floats per partial) non-null: also the softmax statistics at
// `temperature` (typical acceptance).
cudaError_t launch_argmax_partials(const float *logits, int64_t rows, int V, int splits,
                                   float *part_val, int32_t *part_idx, float *part_stats,
                                   float temperature, int32_t *zero_status, int n_zero,
                                   cudaStream_t stream);
// The same partials from `grid` blocks of 512 threads (one warp per chunk at a
// time): the fused step's argmax grid on the SMs of its attention grid's last,
// partial round.
cudaError_t launch_argmax_narrow(const float *logits, int64_t rows, int V, int splits, int grid,
                                 float *part_val, int32_t *part_idx, float *part_stats,
                                 float temperature, int32_t *zero_status, int n_zero,
                                 cudaStream_t stream);
cudaError_t launch_argmax_combine(const float *part_val, const int32_t *part_idx, int64_t rows,
                                  int splits, int32_t *argmax_out, cudaStream_t stream);

struct AcceptArgs {
    const int32_t *cand_tokens;  // [B,T]
    const int32_t *parent;       // [B,T]
    const int32_t *prefix_len;   // [B]
    int32_t *accept_len;         // [B]
    int32_t *path;               // [B,T]
    int32_t *next_token;         // [B]
    int32_t *new_prefix_len;     // [B]
    int32_t *dev_status;         // [B]
    int T, V, S_max;
};

cudaError_t launch_accept_path(const int32_t *argmax, const AcceptArgs &a, int B,
                               cudaStream_t stream);

// Node argmax in one grid, a cluster of CTAs per row; with lse_out also the
// natural-log log-sum-exp and entropy of softmax(row / temperature).
cudaError_t launch_node_argmax(const float *logits, int64_t rows, int V, float temperature,
                               int32_t *argmax_out, float *lse_out, float *ent_out, cudaStream_t stream);

// argmax, natural-log log-sum-exp and entropy per row from stats partials.
cudaError_t launch_node_stats_combine(const float *part_val, const int32_t *part_idx,
                                      const float *part_stats, int64_t rows, int splits,
                                      int32_t *argmax_out, float *lse_out, float *ent_out,
                                      cudaStream_t stream);

cudaError_t launch_typical_accept(const float *logits, const float *lse, const float *ent,
                                  const int32_t *argmax, const AcceptArgs &a, int B,
                                  float temperature, float epsilon, float delta,
                                  cudaStream_t stream);

// chained: as a programmatic dependent of the stream's previous grid.
cudaError_t launch_kv_compact(void *k_cache, void *v_cache, const void *k_tree,
                              const void *v_tree, const int32_t *path,
                              const int32_t *accept_len, const int32_t *prefix_len, int L,
                              int B, int H, int T, int D, int S_max, int elem_bytes,
                              cudaStream_t stream, bool chained = true);

// Next-step candidate tree: at most this many guesses per depth.
constexpr int kNextMaxK = 16;
constexpr int kNextMaxEpt = 128;
constexpr int kNextMaxSplit = 8;    // CTAs (a cluster) sharing one row's columns

cudaError_t launch_next_tree(const float *logits, const int32_t *parent, const int32_t *cand,
                             const int32_t *path, const int32_t *accept_len,
                             const int32_t *next_token, int B, int T, int V, int n_states,
                             int T_next, const int32_t *tmpl_parent, const int32_t *tmpl_rank, int K,
                             int n_ept, int ept_mean, int32_t *topk, int32_t *kstate, float *lse,
                             int num_sms, int32_t *next_parent, int32_t *next_cand,
                             int32_t *next_state, int32_t *status, cudaStream_t stream);

// fp32 -> bf16 copies (round to nearest even) of n tensors [lbh][rows][D]; of a
// `cache` tensor only the rows below the sequence's prefix length.  chained: as
// a programmatic dependent of the stream's previous grid.
struct RoundArgs {
    struct Tensor {
        const float *src;
        uint16_t *dst;
        int rows;
        int cache;
    } t[5];
    const int32_t *prefix_len;
    int n, B, H, D;
};
cudaError_t launch_round_bf16(const RoundArgs &r, int64_t lbh, bool chained, cudaStream_t stream);

// Zero `n` status words once the preceding grid has completed, as a
// programmatic dependent launch that lets the next grid launch at once.
cudaError_t launch_zero_status(int32_t *status, int n, cudaStream_t stream);

// ---- 4-bit cache (ppd_kv4.cuh has the format): slices = L * B * H
struct Kv4AppendParams {
    const void *k_new, *v_new;       // [slices][T][D] bf16 or (f32) fp32
    uint8_t *k_cache, *v_cache;      // [slices][S_max][D / 2]
    uint8_t *k_scale, *v_scale;      // [slices][S_max][D / 32]
    const int32_t *rows;             // [B,T] or null
    const int32_t *start, *n_new;    // [B]
    int32_t *dev_status;             // [B]
    long long slices;
    int B, H, T, D, S_max, f32;
};
cudaError_t launch_kv4_append(const Kv4AppendParams &p, cudaStream_t stream);

struct Kv4ReadParams {
    const uint8_t *cache, *scale;    // K's or V's
    const int32_t *start, *n;        // [B]
    void *out;                       // [slices][N][D] bf16 or fp32
    long long slices;
    int B, H, N, D, S_max, f32;
};
cudaError_t launch_kv4_read(const Kv4ReadParams &p, cudaStream_t stream);

// Attention over a 4-bit cache: query rows of a slice are its G heads' T tokens.
struct Kv4AttnParams {
    const void *q;                   // [slices][G * T][D] bf16 or fp32
    const uint8_t *k_cache, *k_scale, *v_cache, *v_scale;
    const void *k_tree, *v_tree;     // [slices][T][D]
    const int32_t *prefix_len, *parent;
    uint16_t *out;                   // bf16 [slices][G * T][D]
    float *lse;                      // [slices][G * T] or null
    int32_t *dev_status;
    size_t scale_bytes;              // of k_scale, and of v_scale
    long long slices;
    int B, H, G, T, S_max, f32;
    float scale_log2;                // softmax scale * log2(e)
    int splits;                      // parts that a slice's keys are shared out to
    float *part_o;                   // splits > 1: [slices][splits][G * T][D] unnormalised outputs
    float2 *part_ml;                 // [slices][splits][G * T] maxima (log2) and sums
};
cudaError_t launch_kv4_attention(const Kv4AttnParams &p, int D, cudaStream_t stream);

// More query rows: units are blocks of TP rows of a slice (p.n_qb of them, n_tt tiles of tree
// keys each), shared out by their key tiles when p.split, on `grid` CTAs.
inline __host__ __device__ size_t kv4_slot_floats(int D, int TP) { return (size_t)TP * (D + 2); }
cudaError_t launch_kv4_attention_wide(const AttnParams &p, const Kv4AttnParams &x, int D, int TP, int grid, cudaStream_t stream);

// Attention weight of the accepted nodes, added up per cached row.
struct KvWeightParams {
    const void *q;                   // [slices][G][T][D] bf16 or fp32
    const float *lse;                // [slices][G][T]
    const uint8_t *k_cache;          // bf16 rows, or codes with
    const uint8_t *k_scale;          // their scales (null: bf16)
    const void *k_tree;              // [slices][T][D]
    const int32_t *path, *accept_len, *prefix_len;
    float *weight;                   // [slices][S_max]
    long long slices;
    int B, H, G, T, S_max, f32;
    float scale_log2;
    size_t scale_bytes;              // of k_scale
    int splits;                      // blocks of a slice
};
int kv_weight_blocks(bool kv4);   // that an SM holds
cudaError_t launch_kv_weight(const KvWeightParams &p, int D, cudaStream_t stream);

// The rows kept of each slice, and the planes they are rows of.
struct KvPlane {
    const void *src;                 // [slices][S_max][row_bytes]
    void *dst;                       // [slices][S_out][row_bytes]; src: in place
    int row_bytes, unit;             // bytes moved at once: a power of two up to 16
    int parts;                       // blocks of a slice
};
constexpr int kMaxPlanes = 9;        // eight of the caller's, and the weights
struct KvEvictParams {
    const float *weight;             // [slices][S_max]
    const int32_t *length;           // [B]
    int32_t *kept;                   // [slices][budget]
    int32_t *new_len, *dev_status;   // [B]
    long long slices;
    int B, H, S_max, S_out, budget, sink, recent;
    KvPlane plane[kMaxPlanes];
    int planes, move_blocks;         // the planes' parts together
};
cudaError_t launch_kv_evict(const KvEvictParams &p, cudaStream_t stream);

// Drafted tokens verified with given random numbers.
struct SampleParams {
    const float *logits;             // [B,T,V]
    const int32_t *cand, *parent;    // [B,T]
    const int32_t *prefix_len;       // [B]
    const float *draft_probs;        // [B,n_draft,V] or null
    const int32_t *draft_row;        // [B,T] or null
    const float *u;                  // [B,T]
    const float *noise;              // [B,V]
    int32_t *accept_len, *path, *next_token, *new_prefix_len, *dev_status;
    float *accept_prob;              // [B,T] or null
    int B, T, V, S_max, n_draft;
    float k;                         // log2(e) / temperature
    int chunk;                       // logits of a CTA of the cluster (a multiple of 4)
};
// Logits of a CTA at most (its shared memory).
constexpr int kSampleMaxChunk = 48 * 1024;
cudaError_t launch_sample_accept(const SampleParams &p, int cluster, cudaStream_t stream);

// ---- a pool of pages
// Sequences of one ppd_page_assign call (their sums lie in shared memory).
constexpr int kMaxAssign = 8192;
struct PageAssignParams {
    const int32_t *old_len, *new_len, *n_free;   // [B], [B], [1]
    int32_t *table;                  // [B][max_pages]
    int32_t *free_pages;             // [n_pages]
    int32_t *new_n_free, *out_len;   // [1], [B]
    int32_t *slots, *slot_start;     // [max_slots], [B + 1]
    int32_t *dev_status;             // [B]
    int B, page_shift, n_pages, max_pages, max_slots;
    int vec;                         // slots is 16-byte aligned
};
cudaError_t launch_page_assign(const PageAssignParams &p, int num_sms, cudaStream_t stream);

struct PageAppendParams {
    const void *k_new, *v_new;       // [slices][T][D] bf16 or (f32) fp32
    void *k_pages, *v_pages;         // bf16 [L][n_pages][H][page][D]
    const int32_t *slots, *slot_start, *rows;   // rows [B,T] or null
    int32_t *dev_status;             // [B]
    long long slices;
    int B, H, T, D, n_pages, page_shift, max_slots, f32;
    int chunks;                      // blocks of a slice
};
int page_append_chunks(int T);
cudaError_t launch_page_append(PageAppendParams p, cudaStream_t stream);

// ---- log probabilities of given tokens
constexpr int kLogMaxK = 32;
struct LogScale {
    float k;                         // log2(e) / temperature
    float span;                      // 200 / k
    float fused;                     // of maxima m below this in size |m k| < 2^20, and m - span is a number
    float h, kh;                     // 1/2 and 2 k where k < 1, else 1 and k
};
struct LogprobParams {
    const void *logits;              // [B,T,V] fp32 or bf16
    const int32_t *tokens, *rows;    // [B,n]; rows null: row i
    float *logprob, *entropy;        // [B,n]
    int32_t *rank;                   // [B,n]
    int32_t *top_tokens;             // [B,n,K]
    float *top_logprobs;
    int32_t *dev_status;             // [B]
    int B, T, V, n, K, bf16;
    LogScale scale;
    int cluster;                     // CTAs of a row
};
cudaError_t launch_token_logprobs(LogprobParams p, int num_sms, cudaStream_t stream);

cudaError_t launch_selftest_umma(const CUtensorMap &ma, const CUtensorMap &mb, const void *a_raw,
                                 const void *b_raw, float *d, int mode, int N, cudaStream_t stream);

}  // namespace ppd
