// ppd_sample.cu -- drafted tokens of a tree verified against the target's probabilities
// with given random numbers, and the token after the last accepted one drawn from what the
// rejections left.
#include "ppd_device.cuh"

#include <cmath>

namespace ppd {

// A cluster of CTAs per sequence, each with its share of the vocabulary in shared memory.
// The walk starts at the root.  At node j the cluster has R = exp((x - M) / temperature) of
// j's logits x and Z, the sum of R.  Child c (in index order) with token t is accepted when
//     u_c < R_t / (Z q_t),    q the distribution that c was drawn from
// (q_t = 1 for a child that was not drawn but chosen); rejected, it leaves R <- max(R / Z - q, 0)
// (R_t <- 0).  The token after the end node is the first of the largest R_v / E_v: with E_v
// exponentially distributed it is v with probability R_v / Z.
//
// What a chosen child's rejection takes away is one token, so those tokens are left out of
// the sum and of the share from the start and kept as numbers beside it: a node costs
// one pass over its logits and one exchange of the CTAs' maxima and sums, its chosen
// children none; a drawn child's rejection costs one pass over the share and its draft row,
// and an exchange.  Every CTA takes the same decisions from the same numbers.
constexpr int kSampleThreads = 512;

struct SampleShared {
    int par[kMaxTree], tok[kMaxTree], row[kMaxTree];   // parents, tokens, draft rows
    float u[kMaxTree], value[kMaxTree], prob[kMaxTree];   // value: R at the node's token
    int child[kMaxTree];      // children of the node, in order
    int path[kMaxTree];
    float2 part[2][kMaxCluster];
    unsigned long long best[kMaxCluster];
    float warp[kSampleThreads / 32];
    unsigned long long warp_best[kSampleThreads / 32];
    int n_child, verdict;
};

template <class Op>
PPD_DEV float block_reduce(float v, float *warp_s, float none, Op op)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) warp_s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = threadIdx.x % 32 < kSampleThreads / 32 ? warp_s[threadIdx.x % 32] : none;
#pragma unroll
    for (int o = kSampleThreads / 64; o; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
    return __shfl_sync(0xffffffffu, v, 0);
}

__global__ void __launch_bounds__(kSampleThreads, 3) sample_accept_kernel(const SampleParams p, int cluster)
{
    extern __shared__ __align__(16) float e[];   // this CTA's share of R
    __shared__ SampleShared s;
    pdl_release();
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)(blockIdx.x % cluster), b = (int)(blockIdx.x / cluster);
    const int T = p.T, V = p.V;
    const int lo = min(V, rank * p.chunk), n = min(V, lo + p.chunk) - lo;
    const float *x0 = p.logits + (size_t)b * T * V;
    const float *q0 = p.draft_probs ? p.draft_probs + (size_t)b * p.n_draft * V : nullptr;

    // ------------------------------------------------ the tree
    bool bad = false;
    for (int i = tid; i < T; i += kSampleThreads) {
        const int pa = ld_input(p.parent + (size_t)b * T + i), tk = ld_input(p.cand + (size_t)b * T + i);
        const int dr = q0 && p.draft_row ? ld_input(p.draft_row + (size_t)b * T + i) : -1;
        bad |= i == 0 ? (pa != -1 || tk < 0 || tk >= V) : (pa < 0 || pa >= i || tk < -1 || tk >= V);
        bad |= i > 0 && tk >= 0 && (dr < -1 || dr >= p.n_draft);
        s.par[i] = pa;
        s.tok[i] = tk;
        s.row[i] = dr;
        s.u[i] = ld_input(p.u + (size_t)b * T + i);
        s.prob[i] = -1.f;
    }
    bad = __syncthreads_or(bad);
    const int P = ld_input(p.prefix_len + b);
    int err = bad ? kErrTree : (P < 0 || P > p.S_max ? kErrCapacity : kOk);

    int phase = 0;
    float M = 0.f, f = 1.f, Z = 0.f, rest = 0.f;   // R = f e; rest: the sum of R in the shares
    // maxima and sums of the CTAs together: M, this CTA's factor and the sum
    auto exchange = [&](float m_c, float s_c) {
        if (tid < cluster) st_cluster_v2(cluster_map(smem_addr(&s.part[phase][rank]), (uint32_t)tid), m_c, s_c);
        cluster_sync();
        M = -INFINITY;
        for (int r = 0; r < cluster; ++r) M = fmaxf(M, s.part[phase][r].x);
        rest = 0.f;
        for (int r = 0; r < cluster; ++r) {
            const float2 v = s.part[phase][r];
            rest += v.x == -INFINITY ? v.y : v.y * ex2((v.x - M) * p.k);   // y: 0, or NaN
        }
        f = m_c == -INFINITY ? 1.f : ex2((m_c - M) * p.k);
        phase ^= 1;
    };
    auto fmax_op = [](float a, float c) { return fmaxf(a, c); };
    // the node's logits into the share; `leave`: without the chosen children's tokens
    auto load_row = [&](int node, bool leave) {
        const float *x = x0 + (size_t)node * V + lo;
        float m = -INFINITY;
        if ((reinterpret_cast<uintptr_t>(x) & 15) == 0 && (n & 3) == 0) {
            for (int v = tid; v < n / 4; v += kSampleThreads) {
                const float4 a = ld_input(reinterpret_cast<const float4 *>(x) + v);
                reinterpret_cast<float4 *>(e)[v] = a;
                m = fmaxf(m, fmaxf(fmaxf(a.x, a.y), fmaxf(a.z, a.w)));
            }
        } else {
            for (int v = tid; v < n; v += kSampleThreads) {
                const float a = ld_input(x + v);
                e[v] = a;
                m = fmaxf(m, a);
            }
        }
        m = block_reduce(m, s.warp, -INFINITY, fmax_op);
        if (leave) {
            for (int i = tid; i < s.n_child; i += kSampleThreads) {
                const int c = s.child[i], v = s.tok[c] - lo;
                // (a NaN stays where it is: it is what the row is)
                if (s.row[c] < 0 && v >= 0 && v < n && e[v] == e[v]) e[v] = -INFINITY;
            }
            __syncthreads();
        }
        float sum = 0.f;
        const float mm = m == -INFINITY ? 0.f : m;
        for (int v = tid; v < n; v += kSampleThreads) {
            const float r = ex2((e[v] - mm) * p.k);
            e[v] = r;
            sum += r;
        }
        sum = block_reduce(sum, s.warp, 0.f, OpAdd());
        exchange(m, sum);
    };

    int cur = 0, len = 1;
    bool flat = false;   // the end node's logits have no distribution
    if (err == kOk) {
        if (tid == 0) s.path[0] = 0;
        while (true) {
            // the node's children, in order
            __syncthreads();
            if (warp == 0) {
                int k = 0;
                for (int i0 = cur + 1 - (cur + 1) % 32; i0 < T; i0 += 32) {
                    const int i = i0 + lane;
                    const bool is = i > cur && i < T && s.par[i] == cur && s.tok[i] >= 0;
                    const uint32_t all = __ballot_sync(0xffffffffu, is);
                    if (is) s.child[k + __popc(all & ((1u << lane) - 1u))] = i;
                    k += __popc(all);
                }
                if (lane == 0) s.n_child = k;
            }
            __syncthreads();
            const int kids = s.n_child;
            load_row(cur, true);
            // R at the children's tokens; a chosen token counts once, at its first child
            flat = !(M > -INFINITY && M < INFINITY) || rest != rest;
            for (int i = tid; i < kids; i += kSampleThreads)
                s.value[i] = ex2((ld_input(x0 + (size_t)cur * V + s.tok[s.child[i]]) - M) * p.k);
            __syncthreads();
            int next = -1, at = 0;
            while (at < kids) {
                if (warp == 0) {
                    // Z: the shares and what is left of the chosen children's tokens
                    auto chosen_sum = [&]() {
                        float z = 0.f;
                        for (int i = lane; i < kids; i += 32) {
                            const int c = s.child[i];
                            bool first = s.row[c] < 0;
                            for (int h = 0; first && h < i; ++h) first = s.row[s.child[h]] >= 0 || s.tok[s.child[h]] != s.tok[c];
                            if (first) z += s.value[i];
                        }
#pragma unroll
                        for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
                        return z;
                    };
                    int verdict = -1;   // all rejected; i: child i accepted; kMaxTree + i: drawn child i rejected
                    for (; at < kids; ++at) {
                        const int c = s.child[at], t = s.tok[c];
                        const float z = rest + chosen_sum();
                        float a = s.value[at] / z;
                        if (s.row[c] >= 0) {
                            const float q = ld_input(q0 + (size_t)s.row[c] * V + t);
                            a = q > 0.f ? a / q : 0.f;
                        }
                        a = flat || !(z > 0.f) ? 0.f : fminf(a, 1.f);
                        if (lane == 0) s.prob[c] = a;
                        if (s.u[c] < a) {
                            verdict = at;
                            break;
                        }
                        if (flat) continue;
                        if (s.row[c] >= 0) {
                            verdict = kMaxTree + at;
                            break;
                        }
                        __syncwarp();
                        for (int i = lane; i < kids; i += 32)
                            if (s.tok[s.child[i]] == t) s.value[i] = 0.f;
                        __syncwarp();
                    }
                    const float z = rest + chosen_sum();
                    if (lane == 0) {
                        s.verdict = verdict;
                        s.warp[0] = z;
                    }
                }
                __syncthreads();
                const int verdict = s.verdict;
                Z = s.warp[0];
                if (verdict < 0) break;
                if (verdict < kMaxTree) {
                    next = s.child[verdict];
                    break;
                }
                // a drawn child's rejection: what its distribution covers is taken away
                at = verdict - kMaxTree + 1;
                const float *q = q0 + (size_t)s.row[s.child[at - 1]] * V;
                const float zf = f / Z;
                float sum = 0.f;
                for (int v = tid; v < n; v += kSampleThreads) {
                    const float r = fmaxf(e[v] * zf - ld_input(q + lo + v), 0.f);
                    e[v] = r;
                    sum += r;
                }
                for (int i = tid; i < kids; i += kSampleThreads)
                    s.value[i] = fmaxf(s.value[i] / Z - ld_input(q + s.tok[s.child[i]]), 0.f);
                // (e is 0 at the chosen children's tokens, and stays it)
                sum = block_reduce(sum, s.warp, 0.f, OpAdd());
                exchange(0.f, sum);
                __syncthreads();
            }
            if (next < 0) break;
            cur = next;
            if (tid == 0) s.path[len] = cur;
            ++len;
        }
        if ((long long)P + len > p.S_max) err = kErrCapacity;
    }

    // ------------------------------------------------ the next token
    if (err == kOk) {
        // every child was rejected: the shares hold what is left
        const bool none = !flat && !(rest > 0.f);
        if (none) load_row(cur, false);   // nothing left: the node's own distribution
        const float *x = x0 + (size_t)cur * V + lo, *noise = p.noise + (size_t)b * V + lo;
        unsigned long long best = 0;
        for (int v = tid; v < n; v += kSampleThreads) {
            float r;
            if (flat) {   // the first NaN, or the first of the largest
                const float a = ld_input(x + v);
                r = a != a ? 2.f : a == M ? 1.f : 0.f;
            } else {
                r = f * e[v] / ld_input(noise + v);
                if (!(r >= 0.f)) r = 0.f;
            }
            const unsigned long long key = (unsigned long long)__float_as_uint(r) << 32 | (0xFFFFFFFFu - (uint32_t)(lo + v));
            if (key > best) best = key;
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            const unsigned long long y = __shfl_xor_sync(0xffffffffu, best, o);
            if (y > best) best = y;
        }
        if (lane == 0) s.warp_best[warp] = best;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kSampleThreads / 32; ++w)
                if (s.warp_best[w] > best) best = s.warp_best[w];
            st_cluster_u64(cluster_map(smem_addr(&s.best[rank]), 0), best);
        }
        cluster_sync();
        if (rank == 0 && tid == 0) {
            for (int r = 0; r < cluster; ++r)
                if (s.best[r] > best) best = s.best[r];
            p.next_token[b] = (int)(0xFFFFFFFFu - (uint32_t)best);
        }
    }
    if (rank != 0) return;
    __syncthreads();
    const int n_out = err == kOk ? len : 0;
    for (int i = tid; i < T; i += kSampleThreads) {
        p.path[(size_t)b * T + i] = i < n_out ? s.path[i] : -1;
        if (p.accept_prob) p.accept_prob[(size_t)b * T + i] = err == kOk ? s.prob[i] : -1.f;
    }
    if (tid == 0) {
        p.accept_len[b] = n_out;
        p.new_prefix_len[b] = P + n_out;
        p.dev_status[b] = err;
        if (err != kOk) p.next_token[b] = -1;
    }
}

cudaError_t launch_sample_accept(const SampleParams &p, int cluster, cudaStream_t stream)
{
    static std::atomic<uint64_t> configured{0};
    const cudaError_t e = allow_smem(sample_accept_kernel, kSampleMaxChunk * 4, configured);
    if (e != cudaSuccess) return e;
    return launch_chained_smem(sample_accept_kernel, dim3((unsigned)(p.B * cluster)), dim3(kSampleThreads),
                               dim3((unsigned)cluster), (uint32_t)p.chunk * 4u, stream, p, cluster);
}

}  // namespace ppd
