// ppd_attention.cu -- the key-row kernel (ppd_attention_key.cuh) over contiguous caches: its
// instantiations, the merge of units cut by the work split, and the launches.
#include "ppd_attention_key.cuh"

namespace ppd {

// The merge of the units cut by the work split: blockIdx.x is an attention
// CTA (gridDim.x = the attention grid), blockIdx.y a block of 256 / (D / 8)
// rows of the unit that CTA recorded; each thread merges 8 columns of a row,
// once the attention grid has completed.
__global__ void __launch_bounds__(256) split_merge_kernel(const AttnParams p, int D)
{
    // a next grid launched as a programmatic dependent may start at once; it
    // waits for this grid to complete before it reads or writes anything
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const SplitRecord r = p.split_rec[blockIdx.x];
    if (r.u < 0) return;
    const int per_row = D / 8;
    const int rows_per_block = (int)blockDim.x / per_row;
    const int lbh = r.u / p.n_qb, qb = r.u - lbh * p.n_qb;
    const int n_rows = min(kSplitRows, p.T - qb * kSplitRows);
    const int row = (int)blockIdx.y * rows_per_block + (int)threadIdx.x / per_row;
    if (row >= n_rows) return;
    const SplitParts sp = split_parts(r.n_shared, r.off, r.n_tiles);
    split_merge_chunk(p.split_part, p.out, p.lse, sp, r.n_shared, (int)gridDim.x,
                      (size_t)lbh * p.T + (size_t)qb * kSplitRows, row, ((int)threadIdx.x % per_row) * 8, D);
}

cudaError_t launch_split_merge(const AttnParams &p, int D, int grid, cudaStream_t stream)
{
    const int rows_per_block = 256 / (D / 8);
    const int rows = p.T < kSplitRows ? p.T : kSplitRows;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid, (unsigned)((rows + rows_per_block - 1) / rows_per_block));
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, split_merge_kernel, p, D);
}

template <int D, int TP>
static cudaError_t launch_tree_attention_t(const AttnMaps &m, const AttnParams &p, int num_sms,
                                           bool programmatic, cudaStream_t stream)
{
    using Lay = AttnLayout<D, TP>;
    static std::atomic<uint64_t> configured[4] = {{0}, {0}, {0}, {0}};
    if (whole_ragged(p))
        return launch_attention_grid(tree_attention_kernel<D, TP, 3>, Lay::SMEM_BYTES, Lay::THREADS,
                                     configured[3], m, p, num_sms, programmatic, stream);
    if (p.cluster > 1)
        return launch_attention_grid(tree_attention_kernel<D, TP, 2>, Lay::SMEM_BYTES, Lay::THREADS,
                                     configured[2], m, p, num_sms, programmatic, stream);
    if (p.split)
        return launch_attention_grid(tree_attention_kernel<D, TP, 1>, Lay::SMEM_BYTES, Lay::THREADS,
                                     configured[1], m, p, num_sms, programmatic, stream);
    return launch_attention_grid(tree_attention_kernel<D, TP, 0>, Lay::SMEM_BYTES, Lay::THREADS,
                                 configured[0], m, p, num_sms, programmatic, stream);
}

// Asked of one attention kernel for all of them: each takes a whole SM, so the
// answer only depends on how the device groups its SMs.
int max_attention_clusters(int size)
{
    static std::atomic<int> cache[64][kMaxCluster + 1];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    if (dev < 0 || dev >= 64 || size < 1 || size > kMaxCluster) return 0;
    return asked_once(cache[dev][size], [&] {
        using Lay = AttnLayout<128, 64>;
        auto kern = tree_attention_kernel<128, 64, 2>;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)size);
        cfg.blockDim = dim3(Lay::THREADS);
        cfg.dynamicSmemBytes = Lay::SMEM_BYTES;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)size;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Lay::SMEM_BYTES) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) {
            (void)cudaGetLastError();
            return -1;
        }
        return n;
    });
}

cudaError_t launch_tree_attention(const AttnMaps &m, const AttnParams &p, int D, int num_sms,
                                  bool programmatic, cudaStream_t stream)
{
    cudaError_t e;
    if (p.T_pad > 64) e = launch_tree_attention_rows(m, p, D, num_sms, programmatic, stream);
    else if (D == 128 && p.T_pad == 64) e = launch_tree_attention_t<128, 64>(m, p, num_sms, programmatic, stream);
    else if (D == 128) e = launch_tree_attention_t<128, 32>(m, p, num_sms, programmatic, stream);
    else if (p.T_pad == 64) e = launch_tree_attention_t<64, 64>(m, p, num_sms, programmatic, stream);
    else e = launch_tree_attention_t<64, 32>(m, p, num_sms, programmatic, stream);
    if (e != cudaSuccess || !p.split) return e;
    return launch_split_merge(p, D, attention_grid(p, num_sms), stream);
}

}  // namespace ppd
