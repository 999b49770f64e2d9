// ppd_sample.cu -- drafted tokens of a tree verified against the target's probabilities
// with given random numbers, and the token after the last accepted one drawn from what the
// rejections left.
#include "ppd_kv4.cuh"

#include <cmath>
#include <type_traits>

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
//
// Bound by the chain of a walk's passes, not by their bytes (one sequence, 32,000 tokens, chosen
// guesses: 9 us; 80 sequences, 50,257 tokens, drawn: 44 us, the longest of their walks seven or eight
// passes): a thread keeps to its own elements
// of the share and a warp to its own maximum, so that a pass has one barrier of the block and
// one of the cluster; the children's entries are asked for before the row.  (Asking L2 for
// the draft row or the noise ahead of their passes made 80 sequences 42 -> 56 us.)
constexpr int kSampleThreads = 512, kSampleWarps = kSampleThreads / 32;

struct SampleShared {
    int par[kMaxTree], tok[kMaxTree], row[kMaxTree];   // parents, tokens, draft rows
    float u[kMaxTree], prob[kMaxTree];
    int child[kMaxTree];      // children of the node, in order
    float value[kMaxTree];    // R at their tokens
    float draft[kMaxTree];    // q at their tokens
    bool first[kMaxTree];     // a chosen child whose token no chosen one before it has
    int path[kMaxTree];
    float2 warp[kSampleWarps];
    float2 part[2][kMaxCluster];
    unsigned long long best[kMaxCluster], warp_best[kSampleWarps];
    int n_child, verdict, next;
    float z;
};

// VEC: 16-byte accesses, which every row allows (80 sequences of 50,256 tokens: 38 us, by elements
// 42).
template <bool VEC>
__global__ void __launch_bounds__(kSampleThreads, 3) sample_accept_kernel(const SampleParams p, int cluster)
{
    extern __shared__ __align__(16) float e[];   // this CTA's share: R over a factor of the warp
    __shared__ SampleShared s;
    cluster_sync();   // every CTA of the cluster has started before one stores into another's shared memory
    pdl_release();
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)(blockIdx.x % cluster), b = (int)(blockIdx.x / cluster);
    const int T = p.T, V = p.V;
    const int lo = min(V, rank * p.chunk), n = min(V, lo + p.chunk) - lo;
    const float *x0 = p.logits + (size_t)b * T * V + lo;
    const float *q0 = p.draft_probs ? p.draft_probs + (size_t)b * p.n_draft * V + lo : nullptr;
    // a thread's elements are its own throughout
    constexpr int STEP = VEC ? 4 : 1, STRIDE = kSampleThreads * STEP;
    constexpr int AHEAD = VEC ? 2 : 8;
    using Own = std::conditional_t<VEC, float4, float>;
    const int own0 = tid * STEP;
    auto owner = [&](int v) { return v / STEP % kSampleThreads; };

    // ------------------------------------------------ the tree
    bool bad = false;
    for (int i = tid; i < T; i += kSampleThreads) {
        const int pa = ld_input(p.parent + (size_t)b * T + i), tk = ld_input(p.cand + (size_t)b * T + i);
        const int dr = q0 ? ld_input(p.draft_row + (size_t)b * T + i) : -1;
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
    float M = 0.f, f = 1.f, rest = 0.f;   // R = f e; rest: the sum of R in the shares
    // the warps' maxima and sums together: M, this warp's factor and the sum of all
    auto combine = [&](float2 v) {   // over a warp's lanes
        float m = v.x;
#pragma unroll
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        float y = v.x == -INFINITY ? v.y : v.y * ex2((v.x - m) * p.k);   // y: 0, or NaN
#pragma unroll
        for (int o = 16; o; o >>= 1) y += __shfl_xor_sync(0xffffffffu, y, o);
        return make_float2(m, y);
    };
    auto exchange = [&](float m_w, float s_w) {   // (a lane's maximum is its warp's, a sum its own)
#pragma unroll
        for (int o = 16; o; o >>= 1) s_w += __shfl_xor_sync(0xffffffffu, s_w, o);
        if (lane == 0) s.warp[warp] = make_float2(m_w, s_w);
        __syncthreads();
        if (warp == 0) {
            const float2 v = combine(lane < kSampleWarps ? s.warp[lane] : make_float2(-INFINITY, 0.f));
            if (lane < cluster) st_cluster_v2(cluster_map(smem_addr(&s.part[phase][rank]), (uint32_t)lane), v.x, v.y);
        }
        cluster_sync();
        M = -INFINITY;
        for (int r = 0; r < cluster; ++r) M = fmaxf(M, s.part[phase][r].x);
        rest = 0.f;
        for (int r = 0; r < cluster; ++r) {
            const float2 v = s.part[phase][r];
            rest += v.x == -INFINITY ? v.y : v.y * ex2((v.x - M) * p.k);
        }
        f = m_w == -INFINITY ? 1.f : ex2((m_w - M) * p.k);
        phase ^= 1;
    };
    // the node's logits into the share, without the first `leave` children's chosen tokens
    auto load_row = [&](int node, int leave) {
        const float *x = x0 + (size_t)node * V;
        const uint32_t to = smem_addr(e);
#pragma unroll 4
        for (int v = own0; v < n; v += STRIDE) {   // all of a thread's elements on their way at once
            if constexpr (VEC) cp_async16(to + v * 4, x + v, 16u);
            else cp_async4(to + v * 4, x + v, 4u);
        }
        cp_async_commit();
        cp_async_wait<0>();
        float m = -INFINITY;
#pragma unroll 4
        for (int v = own0; v < n; v += STRIDE) {
            if constexpr (VEC) {
                const float4 a = *reinterpret_cast<const float4 *>(e + v);
                m = fmaxf(m, fmaxf(fmaxf(a.x, a.y), fmaxf(a.z, a.w)));
            } else {
                m = fmaxf(m, e[v]);
            }
        }
        for (int i = 0; i < leave; ++i) {
            const int c = s.child[i], v = s.tok[c] - lo;
            // (a NaN stays where it is: it is what the row is)
            if (s.row[c] < 0 && v >= 0 && v < n && owner(v) == tid && e[v] == e[v]) e[v] = -INFINITY;
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float mm = m == -INFINITY ? 0.f : m;
        float sum = 0.f;
#pragma unroll 4
        for (int v = own0; v < n; v += STRIDE) {
            if constexpr (VEC) {
                float4 a = *reinterpret_cast<const float4 *>(e + v);
                a = make_float4(ex2((a.x - mm) * p.k), ex2((a.y - mm) * p.k), ex2((a.z - mm) * p.k), ex2((a.w - mm) * p.k));
                *reinterpret_cast<float4 *>(e + v) = a;
                sum += (a.x + a.y) + (a.z + a.w);
            } else {
                const float r = ex2((e[v] - mm) * p.k);
                e[v] = r;
                sum += r;
            }
        }
        exchange(m, sum);
    };

    int cur = 0, len = 1;
    bool flat = false;   // the end node's logits have no distribution
    if (err == kOk) {
        if (tid == 0) s.path[0] = 0;
        while (true) {
            // the node's children, in order
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
            // their entries of the row and of their draft rows (one each, from thread i)
            float kid_x = 0.f, kid_q = 1.f;
            if (tid < kids) {
                const int c = s.child[tid], t = s.tok[c], r = s.row[c];
                kid_x = ld_input(x0 - lo + (size_t)cur * V + t);
                if (r >= 0) kid_q = ld_input(q0 - lo + (size_t)r * V + t);
                bool first = r < 0;
                for (int h = 0; first && h < tid; ++h) first = s.row[s.child[h]] >= 0 || s.tok[s.child[h]] != t;
                s.first[tid] = first;
            }
            load_row(cur, kids);
            // R at the children's tokens; a chosen token counts once, at its first child
            flat = !(M > -INFINITY && M < INFINITY) || rest != rest;
            if (tid < kids) {
                s.value[tid] = ex2((kid_x - M) * p.k);
                s.draft[tid] = kid_q;
            }
            __syncthreads();
            int next = -1, at = 0;
            while (at < kids) {
                if (warp == 0) {
                    // Z: the shares and what is left of the chosen children's tokens
                    auto chosen_sum = [&]() {
                        float z = 0.f;
                        for (int i = lane; i < kids; i += 32)
                            if (s.first[i]) z += s.value[i];
#pragma unroll
                        for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
                        return z;
                    };
                    int verdict = -1;   // all rejected; i: child i accepted; kMaxTree + i: drawn child i rejected
                    float z = rest + chosen_sum();
                    for (; at < kids; ++at) {
                        const int c = s.child[at], t = s.tok[c];
                        float a = s.value[at] / z;
                        if (s.row[c] >= 0) a = s.draft[at] > 0.f ? a / s.draft[at] : 0.f;
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
                        z = rest + chosen_sum();
                    }
                    if (lane == 0) {
                        s.verdict = verdict;
                        if (verdict >= 0 && verdict < kMaxTree) s.next = s.child[verdict];   // (the list is the next node's soon)
                        s.z = z;
                    }
                }
                __syncthreads();
                const int verdict = s.verdict;
                const float Z = s.z;
                if (verdict < 0) break;
                if (verdict < kMaxTree) {
                    next = s.next;
                    break;
                }
                // a drawn child's rejection: what its distribution covers is taken away
                // (e is 0 at the chosen children's tokens, and stays it)
                at = verdict - kMaxTree + 1;
                const float *q = q0 + (size_t)s.row[s.child[at - 1]] * V;
                if (tid < kids) kid_q = ld_input(q - lo + s.tok[s.child[tid]]);
                const float zf = f / Z;
                float sum = 0.f;
                for (int v0 = own0; v0 < n; v0 += AHEAD * STRIDE) {
                    Own y[AHEAD];   // the loads of several elements in flight
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i)
                        if (v0 + i * STRIDE < n) y[i] = ld_input(reinterpret_cast<const Own *>(q + v0 + i * STRIDE));
#pragma unroll
                    for (int i = 0; i < AHEAD; ++i) {
                        const int v = v0 + i * STRIDE;
                        if (v >= n) break;
                        if constexpr (VEC) {
                            const float4 x = *reinterpret_cast<const float4 *>(e + v);
                            const float4 r = make_float4(fmaxf(x.x * zf - y[i].x, 0.f), fmaxf(x.y * zf - y[i].y, 0.f), fmaxf(x.z * zf - y[i].z, 0.f),
                                                         fmaxf(x.w * zf - y[i].w, 0.f));
                            *reinterpret_cast<float4 *>(e + v) = r;
                            sum += (r.x + r.y) + (r.z + r.w);
                        } else {
                            const float r = fmaxf(e[v] * zf - y[i], 0.f);
                            e[v] = r;
                            sum += r;
                        }
                    }
                }
                if (tid < kids) s.value[tid] = fmaxf(s.value[tid] / Z - kid_q, 0.f);
                exchange(0.f, sum);
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
        if (none) load_row(cur, 0);   // nothing left: the node's own distribution
        const float *x = x0 + (size_t)cur * V, *noise = p.noise + (size_t)b * V + lo;
        unsigned long long best = 0;
        // a thread's best so far; its elements come in ascending order, so the first of equals stays
        float top = -1.f;
        int at = 0;
        auto consider = [&](int v, float r) {
            if (r > top) top = r, at = v;
        };
        // a thread's own elements: the warp's factor is theirs
        const bool wide = VEC && (reinterpret_cast<uintptr_t>(noise) & 15) == 0;
        if (flat)   // the first NaN, or the first of the largest
            for (int v = own0; v < n; v += STRIDE)
                for (int k = 0; k < STEP; ++k) {
                    const float a = ld_input(x + v + k);
                    consider(v + k, a != a ? 2.f : a == M ? 1.f : 0.f);
                }
        // a quotient to two units in the last place, equal for equal sides: an IEEE one took a
        // tenth of a batch's time.  (One that is no number never wins: 0 does where nothing else.)
        for (int v0 = own0; v0 < n && !flat; v0 += AHEAD * STRIDE) {
            float y[AHEAD * STEP];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int v = v0 + i * STRIDE;
                if (v >= n) break;
                if (wide) {
                    const float4 a = ld_input(reinterpret_cast<const float4 *>(noise + v));
                    y[i * STEP] = a.x, y[(i * STEP + 1) % (AHEAD * STEP)] = a.y, y[(i * STEP + 2) % (AHEAD * STEP)] = a.z, y[(i * STEP + 3) % (AHEAD * STEP)] = a.w;
                } else {
#pragma unroll
                    for (int k = 0; k < STEP; ++k) y[i * STEP + k] = ld_input(noise + v + k);
                }
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
#pragma unroll
                for (int k = 0; k < STEP; ++k)
                    if (v0 + i * STRIDE < n) consider(v0 + i * STRIDE + k, __fdividef(f * e[v0 + i * STRIDE + k], y[i * STEP + k]));
        }
        if (own0 < n) {
            if (top < 0.f) top = 0.f, at = own0;
            best = (unsigned long long)__float_as_uint(top) << 32 | (0xFFFFFFFFu - (uint32_t)(lo + at));
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            const unsigned long long y = __shfl_xor_sync(0xffffffffu, best, o);
            if (y > best) best = y;
        }
        if (lane == 0) s.warp_best[warp] = best;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kSampleWarps; ++w)
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
    // (a failed sequence: every CTA has read its inputs before one writes an output in their place)
    if (err != kOk) cluster_sync();
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

template <bool VEC>
static cudaError_t launch_sample_t(const SampleParams &p, int cluster, cudaStream_t stream)
{
    static std::atomic<uint64_t> configured{0};
    const cudaError_t e = allow_smem(sample_accept_kernel<VEC>, kSampleMaxChunk * 4, configured);
    if (e != cudaSuccess) return e;
    return launch_chained_smem(sample_accept_kernel<VEC>, dim3((unsigned)(p.B * cluster)), dim3(kSampleThreads), dim3((unsigned)cluster),
                               (uint32_t)p.chunk * 4u, stream, p, cluster);
}

cudaError_t launch_sample_accept(const SampleParams &p, int cluster, cudaStream_t stream)
{
    const bool vec = p.V % 4 == 0 && (reinterpret_cast<uintptr_t>(p.logits) & 15) == 0 && (reinterpret_cast<uintptr_t>(p.draft_probs) & 15) == 0;
    return vec ? launch_sample_t<true>(p, cluster, stream) : launch_sample_t<false>(p, cluster, stream);
}

}  // namespace ppd
