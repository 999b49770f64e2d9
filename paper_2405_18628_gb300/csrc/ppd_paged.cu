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
// 5.5 us longer, of a call's 67.7).
template <int kRows>
__global__ void __launch_bounds__(256) paged_merge_kernel(const PagedParams p, int D)
{
    __shared__ SplitRecord s_rec;
    __shared__ SplitParts s_parts;
    pdl_release();
    pdl_wait();
    if (threadIdx.x == 0) {
        s_rec = p.split_rec[blockIdx.x];
        if (s_rec.u >= 0) s_parts = split_parts(s_rec.n_shared, s_rec.off, s_rec.n_tiles);
    }
    __syncthreads();
    if (s_rec.u < 0) return;
    const int per_row = D / 8;
    const int lbh = s_rec.u / p.n_qb, qb = s_rec.u - lbh * p.n_qb;
    const int n_rows = min(kRows, p.rows - qb * kRows);
    const int row = (int)(blockIdx.y * (blockDim.x / per_row) + threadIdx.x / per_row);
    if (row >= n_rows) return;
    split_merge_chunk<__nv_bfloat16, kRows, kRows == kSplitRows ? 4 : 2>(
        p.split_part, reinterpret_cast<__nv_bfloat16 *>(p.out), p.lse, s_parts, s_rec.n_shared, (int)gridDim.x,
        (size_t)lbh * p.rows + (size_t)qb * kRows, row, ((int)threadIdx.x % per_row) * 8, D);
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
    const int most = p.pair_units ? 2 * kSplitRows : kSplitRows, rows = p.rows < most ? p.rows : most, per_block = 256 / (D / 8);
    const dim3 grid((unsigned)attention_grid(p, num_sms), (unsigned)((rows + per_block - 1) / per_block));
    return p.pair_units ? launch_chained(paged_merge_kernel<2 * kSplitRows>, grid, dim3(256), dim3(1), stream, p, D)
                        : launch_chained(paged_merge_kernel<kSplitRows>, grid, dim3(256), dim3(1), stream, p, D);
}

}  // namespace ppd
