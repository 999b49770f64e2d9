// ppd_attention_rows.cu -- the query-row kernel (ppd_attention_rows.cuh) over contiguous
// caches: its instantiations and launches.
#include "ppd_attention_rows.cuh"

namespace ppd {

template <int D>
static cudaError_t launch_rows_t(const AttnMaps &m, const AttnParams &p, int num_sms,
                                 bool programmatic, cudaStream_t stream)
{
    static std::atomic<uint64_t> configured[4] = {{0}, {0}, {0}, {0}};
    if (whole_ragged(p))
        return launch_attention_grid(tree_attention_rows_kernel<D, 3>, RowsLayout<D>::SMEM_BYTES, 384,
                                     configured[3], m, p, num_sms, programmatic, stream);
    if (p.cluster > 1)
        return launch_attention_grid(tree_attention_rows_kernel<D, 2>, RowsLayout<D>::SMEM_BYTES, 384,
                                     configured[2], m, p, num_sms, programmatic, stream);
    if (p.split)
        return launch_attention_grid(tree_attention_rows_kernel<D, 1>, RowsLayout<D>::SMEM_BYTES, 384,
                                     configured[1], m, p, num_sms, programmatic, stream);
    return launch_attention_grid(tree_attention_rows_kernel<D, 0>, RowsLayout<D>::SMEM_BYTES, 384,
                                 configured[0], m, p, num_sms, programmatic, stream);
}

cudaError_t launch_tree_attention_rows(const AttnMaps &m, const AttnParams &p, int D, int num_sms,
                                       bool programmatic, cudaStream_t stream)
{
    if (D == 128) return launch_rows_t<128>(m, p, num_sms, programmatic, stream);
    return launch_rows_t<64>(m, p, num_sms, programmatic, stream);
}

}  // namespace ppd
