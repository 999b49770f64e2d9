// ppd_paged.cu -- tree attention over a cache in pages: the key-row kernel
// (ppd_attention_key.cuh) with a producer that copies tiles page by page, for slices of up to 64
// query rows (a row is a tree node of one of the G heads that share the K/V head); the merge
// of units cut by the work split; and the launches.  Slices of more rows run the query-row kernel
// (ppd_paged_rows.cu).
#include "ppd_attention_key.cuh"

namespace ppd {

// The merge of the units cut by the work split, as split_merge_kernel, bf16 out; kRows rows a unit.
// One thread of a block finds the unit's parts, and a thread reads four at a time, two of units of 256
// rows, which have few parts each (every thread by itself, and eight at a time: 96 units of 256 rows took
// 5.5 us longer, of a call's 67.7).  Where a unit has few rows and many parts (a long request's token),
// the block's other threads take parts too and their states are joined in order (two slices
// of 64,000 rows, 4 query rows each, 34.6 -> 23.2 us, one with 8 44.2 -> 29.5).
constexpr int kMergeThreads = 512;   // at most
template <int kRows>
__global__ void __launch_bounds__(kMergeThreads) paged_merge_kernel(const PagedParams p, int D)
{
    constexpr int PB = kRows == kSplitRows ? 4 : 2;
    __shared__ SplitRecord s_rec;
    __shared__ SplitParts s_parts;
    __shared__ float s_join[kRows == kSplitRows ? 10 : 1][kMergeThreads];   // [M, Ls, acc][thread]
    pdl_release();
    pdl_wait();
    if (threadIdx.x == 0) {
        s_rec = p.split_rec[blockIdx.x];
        if (s_rec.u >= 0) s_parts = split_parts(s_rec.n_shared, s_rec.off, s_rec.n_tiles);
    }
    __syncthreads();
    if (s_rec.u < 0) return;
    const int per_row = D / 8, G = (int)gridDim.x, per_block = (int)blockDim.x / per_row;
    const int lbh = s_rec.u / p.n_qb, qb = s_rec.u - lbh * p.n_qb;
    const int n_rows = min(kRows, p.rows - qb * kRows);
    int row = (int)blockIdx.y * per_block + (int)threadIdx.x / per_row;
    const int c0 = ((int)threadIdx.x % per_row) * 8;
    __nv_bfloat16 *out = reinterpret_cast<__nv_bfloat16 *>(p.out);
    const size_t row0 = (size_t)lbh * p.rows + (size_t)qb * kRows;
    if constexpr (kRows == kSplitRows) {
        const int n_parts = s_parts.c_b - s_parts.c_a + 1;
        const int ways = min(per_block / n_rows, (n_parts + PB - 1) / PB);
        if (ways > 1) {   // (the same for the block, whose first is the only one)
            const int way = row / n_rows, share = (n_parts + ways - 1) / ways;
            row -= way * n_rows;
            MergeState st;
            if (way < ways) {
                const int a = s_parts.c_a + way * share;
                st = split_merge_parts<kRows, PB>(p.split_part, s_parts, a, min(s_parts.c_b, a + share - 1), s_rec.n_shared, G, row, c0, D);
            }
            s_join[0][threadIdx.x] = st.M, s_join[1][threadIdx.x] = st.Ls;
#pragma unroll
            for (int x = 0; x < 8; ++x) s_join[2 + x][threadIdx.x] = st.acc[x];
            __syncthreads();
            if (way != 0) return;
            for (int w = 1; w < ways; ++w) {
                const int t = (int)threadIdx.x + w * n_rows * per_row;
                const float m = s_join[0][t];
                if (m == -INFINITY) continue;
                const float Mn = fmaxf(st.M, m), so = ex2(st.M - Mn), wt = ex2(m - Mn);
                st.Ls = fmaf(st.Ls, so, wt * s_join[1][t]);
#pragma unroll
                for (int x = 0; x < 8; ++x) st.acc[x] = fmaf(st.acc[x], so, wt * s_join[2 + x][t]);
                st.M = Mn;
            }
            split_merge_store(st, out, p.lse, row0, row, c0, D);
            return;
        }
    }
    if (row >= n_rows) return;
    split_merge_chunk<__nv_bfloat16, kRows, PB>(p.split_part, out, p.lse, s_parts, s_rec.n_shared, G, row0, row, c0, D);
}

template <int D, int TP>
static cudaError_t launch_paged_t(const AttnMaps &m, const PagedParams &p, int num_sms, cudaStream_t stream)
{
    using Lay = AttnLayout<D, TP>;
    static std::atomic<uint64_t> configured[4] = {{0}, {0}, {0}, {0}};
    const int mode = whole_ragged(p) ? 3 : (p.cluster > 1 ? 2 : (p.split ? 1 : 0));
    auto *kern = tree_attention_kernel<D, TP, 0, true>;
    if (mode == 1) kern = tree_attention_kernel<D, TP, 1, true>;
    if (mode == 2) kern = tree_attention_kernel<D, TP, 2, true>;
    if (mode == 3) kern = tree_attention_kernel<D, TP, 3, true>;
    return launch_attention_grid(kern, Lay::SMEM_BYTES, Lay::THREADS, configured[mode], m, p, num_sms, true, stream);
}

cudaError_t launch_paged_attention(const AttnMaps &m, const PagedParams &p, int D, int num_sms, cudaStream_t stream)
{
    cudaError_t e;
    if (p.T_pad > 64) e = launch_paged_attention_rows(m, p, D, num_sms, stream);
    else if (D == 128) e = p.T_pad == 64 ? launch_paged_t<128, 64>(m, p, num_sms, stream) : launch_paged_t<128, 32>(m, p, num_sms, stream);
    else e = p.T_pad == 64 ? launch_paged_t<64, 64>(m, p, num_sms, stream) : launch_paged_t<64, 32>(m, p, num_sms, stream);
    if (e != cudaSuccess || !p.split) return e;
    const int most = p.pair_units ? 2 * kSplitRows : kSplitRows, rows = p.rows < most ? p.rows : most;
    const int threads = paged_merge_threads(rows, p.n_units, attention_grid(p, num_sms)), per_block = threads / (D / 8);
    const dim3 grid((unsigned)attention_grid(p, num_sms), (unsigned)((rows + per_block - 1) / per_block));
    return p.pair_units ? launch_chained(paged_merge_kernel<2 * kSplitRows>, grid, dim3((unsigned)threads), dim3(1), stream, p, D)
                        : launch_chained(paged_merge_kernel<kSplitRows>, grid, dim3((unsigned)threads), dim3(1), stream, p, D);
}

}  // namespace ppd
