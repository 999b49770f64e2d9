// ppd_paged_rows.cu -- tree attention over a cache in pages for slices of more than 64 query
// rows: the query-row kernel (ppd_attention_rows.cuh) with a producer that copies tiles page by
// page, and its launches.
#include "ppd_attention_rows.cuh"

namespace ppd {

template <int D>
static cudaError_t launch_paged_rows_t(const AttnMaps &m, const PagedParams &p, int num_sms, cudaStream_t stream)
{
    static std::atomic<uint64_t> configured[4] = {{0}, {0}, {0}, {0}};
    const int mode = whole_ragged(p) ? 3 : (p.cluster > 1 ? 2 : (p.split ? 1 : 0));
    auto *kern = tree_attention_rows_kernel<D, 0, true>;
    if (mode == 1) kern = tree_attention_rows_kernel<D, 1, true>;
    if (mode == 2) kern = tree_attention_rows_kernel<D, 2, true>;
    if (mode == 3) kern = tree_attention_rows_kernel<D, 3, true>;
    return launch_attention_grid(kern, RowsLayout<D>::SMEM_BYTES, 384, configured[mode], m, p, num_sms, true, stream);
}

cudaError_t launch_paged_attention_rows(const AttnMaps &m, const PagedParams &p, int D, int num_sms, cudaStream_t stream)
{
    return D == 128 ? launch_paged_rows_t<128>(m, p, num_sms, stream) : launch_paged_rows_t<64>(m, p, num_sms, stream);
}

}  // namespace ppd
