// ppd_logprobs.cu -- log probabilities of given tokens, with entropy, rank and the top
// alternatives (ppd_token_logprobs): what a server answers with beside tokens.
//
// With p = softmax(x / temperature) of an asked row x and t its token, one pass over the row gives
//     m = max x,   s = sum 2^(k (x - m)),   u = sum 2^(k (x - m)) k (x - m),   k = log2(e) / temperature
//     log p_t = (k (x_t - m) - log2 s) ln 2,   entropy = (log2 s - u / s) ln 2
//     rank = entries better than t (NaN first, then the larger value, then the lower index)
// and the K best entries.  A row is taken by a cluster of CTAs (one where there are many rows),
// each streaming its columns in batches of 16-byte loads, the next batch's on their way while
// one is worked on.
//
// The K best: `list` holds the best entries of the batches before, `least` the last of them.  A
// batch in which no thread sees a better entry costs one barrier.  Where up to kFewThreads see
// some, these push all of theirs; where more do (the first batch; rows that rise), the K-th best
// of the maxima of groups of four threads bounds the batch's K-th best from below, and the K
// groups above it push.  A pushed entry's place is the number of better ones.
#include "ppd_device.cuh"
#include "ppd_kernels.h"

#include <climits>
#include <cmath>

namespace ppd {

constexpr int kLogThreads = 256, kLogWarps = kLogThreads / 32;
constexpr int kLogLoads = 4;                   // 16-byte loads of a batch and thread
constexpr int kGroups = kLogThreads / 4;
constexpr int kFewThreads = 64;
static_assert(kLogMaxK <= kGroups, "the K-th best group exists");

PPD_DEV uint32_t order_key(float x)
{
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t u = x == 0.f ? 0u : __float_as_uint(x);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
PPD_DEV float key_value(uint32_t k)
{
    if (k == 0xFFFFFFFFu) return NAN;
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}
PPD_DEV unsigned long long order_entry(uint32_t key, int i) { return (unsigned long long)key << 32 | (uint32_t)~i; }

// Running statistics over entries; bad: a NaN or +inf.
struct RowStats {
    float m, s, u;
    int better, bad;
};

PPD_DEV void merge_stats(RowStats &a, const RowStats &o, float k)
{
    const float nm = fmaxf(a.m, o.m);
    if (nm > -INFINITY) {
        // 2^d (s, u + d s) with d = k (m - nm) <= 0; nothing where there was no entry
        const float da = fmaxf((a.m - nm) * k, -200.f), db = fmaxf((o.m - nm) * k, -200.f);
        const float wa = a.m > -INFINITY ? ex2(da) : 0.f, wb = o.m > -INFINITY ? ex2(db) : 0.f;
        a.u = wa * fmaf(da, a.s, a.u) + wb * fmaf(db, o.s, o.u);
        a.s = wa * a.s + wb * o.s;
    }
    a.m = nm;
    a.better += o.better;
    a.bad |= o.bad;
}

template <bool BF16>
__global__ void __launch_bounds__(kLogThreads, 3) token_logprobs_kernel(const LogprobParams p)
{
    constexpr int E = BF16 ? 8 : 4;            // entries of a load
    constexpr int NV = E * kLogLoads;          // of a batch and thread
    constexpr int kMaxPush = (4 * kLogMaxK > kFewThreads ? 4 * kLogMaxK : kFewThreads) * NV;
    constexpr int eb = BF16 ? 2 : 4;
    __shared__ unsigned long long s_push[kMaxPush], s_list[2][kLogMaxK], s_group[kGroups], s_bound;
    __shared__ RowStats s_stats[kLogWarps], s_cta;
    __shared__ int s_n;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, K = p.K, V = p.V;
    const int rank = (int)blockIdx.x % p.cluster;
    const int item = (int)blockIdx.x / p.cluster;
    const int b = item / p.n, i = item - b * p.n;
    pdl_wait();
    pdl_release();

    // ---- what is asked (the same for the whole cluster); a sequence's status by its first item's CTA
    auto row_of = [&](int it, int at) { return p.rows ? ld_input(p.rows + it) : at; };
    auto outside = [&](int r, int t) { return r < -1 || r >= p.T || t < -1 || t >= V; };
    if (i == 0 && rank == 0) {
        bool any = false;
        for (int x = tid; x < p.n; x += kLogThreads) any |= outside(row_of(item + x, x), ld_input(p.tokens + item + x));
        any = __syncthreads_or(any);
        if (tid == 0) p.dev_status[b] = any ? kErrTree : kOk;
    }
    const int row = row_of(item, i), token = ld_input(p.tokens + item);
    const bool wrong = outside(row, token);
    const bool none = wrong || row < 0;
    if (none) {
        if (rank == 0) {
            if (tid == 0) {
                p.logprob[item] = 0.f;
                p.entropy[item] = 0.f;
                p.rank[item] = -1;
            }
            for (int x = tid; x < K; x += kLogThreads) {
                p.top_tokens[(size_t)item * K + x] = -1;
                p.top_logprobs[(size_t)item * K + x] = 0.f;
            }
        }
        return;   // uniform over the cluster
    }
    const char *x0 = static_cast<const char *>(p.logits) + ((size_t)b * p.T + row) * V * eb;
    auto entry_at = [&](int c) {
        if (BF16) return __uint_as_float((uint32_t)*reinterpret_cast<const volatile uint16_t *>(x0 + (size_t)c * 2) << 16);
        return ld_input(reinterpret_cast<const float *>(x0) + c);
    };
    const float xt = token >= 0 ? entry_at(token) : 0.f;
    const uint32_t kt = order_key(xt);

    // ---- groups of E entries on 16 bytes: group g holds columns [g E - skew, ...)
    const int skew = (int)(reinterpret_cast<uintptr_t>(x0) & 15) / eb;
    const int groups = (int)(((long long)V + skew + E - 1) / E);
    const int g0 = (int)((long long)groups * rank / p.cluster), g1 = (int)((long long)groups * (rank + 1) / p.cluster);
    auto load = [&](int g, uint4 &r) {
        if (g >= g1) return;
        const long long c = (long long)g * E - skew;
        if (c >= 0 && c + E <= V) {
            r = ld_input(reinterpret_cast<const uint4 *>(x0 + c * eb));
            return;
        }
        uint32_t w[4] = {0u, 0u, 0u, 0u};   // a row's ends: the entries that it has
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (c + e < 0 || c + e >= V) continue;
            const uint32_t v = __float_as_uint(entry_at((int)(c + e)));
            if (BF16) w[e / 2] |= (e & 1) ? v : v >> 16;
            else w[e] = v;
        }
        r = make_uint4(w[0], w[1], w[2], w[3]);
    };

    RowStats st{-INFINITY, 0.f, 0.f, 0, 0};
    int cur = 0;   // the list in use
    if (tid < kLogMaxK) s_list[0][tid] = s_list[1][tid] = 0;
    if (tid == 0) s_n = 0;
    __syncthreads();
    unsigned long long least = 0;   // the list's last: entries must be better

    uint4 next[kLogLoads];
#pragma unroll
    for (int q = 0; q < kLogLoads; ++q) load(g0 + q * kLogThreads + tid, next[q]);
    for (int base = g0; base < g1; base += kLogLoads * kLogThreads) {
        float x[NV];
        // entry e of this thread: column col(e), absent outside [0, V) or past the CTA's groups
        auto col = [&](int e) { return (long long)(base + (e / E) * kLogThreads + tid) * E - skew + e % E; };
        auto live = [&](int e) { return base + (e / E) * kLogThreads + tid < g1 && col(e) >= 0 && col(e) < V; };
#pragma unroll
        for (int q = 0; q < kLogLoads; ++q) {
            const uint32_t w[4] = {next[q].x, next[q].y, next[q].z, next[q].w};
#pragma unroll
            for (int e = 0; e < E; ++e)
                x[q * E + e] = BF16 ? __uint_as_float((e & 1) ? (w[e / 2] & 0xFFFF0000u) : (w[e / 2] << 16)) : __uint_as_float(w[e]);
        }
#pragma unroll
        for (int q = 0; q < kLogLoads; ++q) load(base + (kLogLoads + q) * kLogThreads + tid, next[q]);

        // ---- statistics
        float mb = -INFINITY;
        unsigned long long top = 0;
#pragma unroll
        for (int e = 0; e < NV; ++e) {
            if (!live(e)) {
                x[e] = -INFINITY;
                continue;
            }
            const uint32_t key = order_key(x[e]);
            const unsigned long long en = order_entry(key, (int)col(e));
            top = en > top ? en : top;
            st.bad |= x[e] != x[e] || x[e] == INFINITY;
            st.better += en > order_entry(kt, token);
            mb = fmaxf(mb, x[e]);
        }
        if (mb > st.m) {
            RowStats to{mb, 0.f, 0.f, 0, 0};
            merge_stats(st, to, p.k);
        }
        const float m = st.m > -INFINITY ? st.m : 0.f;
#pragma unroll
        for (int e = 0; e < NV; ++e) {
            const float d = fmaxf((x[e] - m) * p.k, -200.f);   // (2^-200 is 0; nothing times an infinity)
            const float v = ex2(d);
            st.s += v;
            st.u = fmaf(v, d, st.u);
        }
        if (K == 0) continue;

        // ---- the K best
        unsigned long long bound = least + 1;
        const int seeing = __syncthreads_count(top >= bound);
        if (seeing == 0) continue;
        if (seeing > kFewThreads) {
            unsigned long long gm = top;
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                const unsigned long long y = __shfl_xor_sync(0xffffffffu, gm, o);
                gm = y > gm ? y : gm;
            }
            if ((lane & 3) == 0) s_group[tid >> 2] = gm;
            if (tid == 0) s_bound = 0;
            __syncthreads();
            if (tid < kGroups) {
                const unsigned long long g = s_group[tid];
                int place = 0;
                for (int y = 0; y < kGroups; ++y) place += s_group[y] > g;
                if (g != 0 && place == K - 1) s_bound = g;   // (fewer groups than K: no bound)
            }
            __syncthreads();
            bound = s_bound > bound ? s_bound : bound;
        }
        if (top >= bound) {
#pragma unroll
            for (int e = 0; e < NV; ++e) {
                if (!live(e)) continue;
                const unsigned long long en = order_entry(order_key(x[e]), (int)col(e));
                if (en >= bound) s_push[atomicAdd(&s_n, 1)] = en;
            }
        }
        if (tid < kLogMaxK) s_list[cur ^ 1][tid] = 0;
        __syncthreads();
        const int n = s_n;
        for (int y = tid; y < n + K; y += kLogThreads) {
            const unsigned long long mine = y < n ? s_push[y] : s_list[cur][y - n];
            int place = 0;
            for (int z = 0; z < n; ++z) place += s_push[z] > mine;
            for (int z = 0; z < K; ++z) place += s_list[cur][z] > mine;
            if (mine != 0 && place < K) s_list[cur ^ 1][place] = mine;
        }
        __syncthreads();
        cur ^= 1;
        least = s_list[cur][K - 1];
        if (tid == 0) s_n = 0;
    }

    // ---- the CTA's statistics, then the cluster's
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        RowStats y;
        y.m = __shfl_xor_sync(0xffffffffu, st.m, o);
        y.s = __shfl_xor_sync(0xffffffffu, st.s, o);
        y.u = __shfl_xor_sync(0xffffffffu, st.u, o);
        y.better = __shfl_xor_sync(0xffffffffu, st.better, o);
        y.bad = __shfl_xor_sync(0xffffffffu, st.bad, o);
        merge_stats(st, y, p.k);
    }
    if (lane == 0) s_stats[warp] = st;
    if (cur == 1 && tid < K) s_list[0][tid] = s_list[1][tid];
    __syncthreads();
    if (tid == 0) {
        st = s_stats[0];
        for (int w = 1; w < kLogWarps; ++w) merge_stats(st, s_stats[w], p.k);
        s_cta = st;
    }
    if (p.cluster > 1) cluster_sync();
    else __syncthreads();
    if (rank == 0) {
        // every thread the whole row's statistics
        st = s_cta;
        for (int c = 1; c < p.cluster; ++c) {
            const uint32_t a = cluster_map(smem_addr(&s_cta), c);
            RowStats y;
            y.m = ld_cluster_f32(a);
            y.s = ld_cluster_f32(a + 4);
            y.u = ld_cluster_f32(a + 8);
            y.better = __float_as_int(ld_cluster_f32(a + 12));
            y.bad = __float_as_int(ld_cluster_f32(a + 16));
            merge_stats(st, y, p.k);
        }
        const bool bad = st.bad || st.m == -INFINITY;
        const float lg = lg2(st.s), ln2 = 0.69314718055994530942f;
        auto logprob = [&](float x) { return bad ? NAN : ((x - st.m) * p.k - lg) * ln2; };
        if (tid == 0) {
            p.logprob[item] = token < 0 ? 0.f : logprob(xt);
            p.entropy[item] = bad ? NAN : (lg - st.u / st.s) * ln2;
            p.rank[item] = token < 0 ? -1 : st.better;
        }
        // the CTAs' lists together: an entry's place is the number of better ones
        const int n = p.cluster * K;
        for (int y = tid; y < n; y += kLogThreads)
            s_push[y] = y < K ? s_list[0][y] : ld_cluster_u64(cluster_map(smem_addr(&s_list[0][0]) + (uint32_t)(y % K) * 8, y / K));
        __syncthreads();
        for (int y = tid; y < n; y += kLogThreads) {
            const unsigned long long mine = s_push[y];
            int place = 0;
            for (int z = 0; z < n; ++z) place += s_push[z] > mine;
            if (mine != 0 && place < K) {
                p.top_tokens[(size_t)item * K + place] = (int)~(uint32_t)mine;
                p.top_logprobs[(size_t)item * K + place] = logprob(key_value((uint32_t)(mine >> 32)));
            }
        }
    }
    if (p.cluster > 1) cluster_sync();   // no list that a peer reads goes away
}

cudaError_t launch_token_logprobs(LogprobParams p, int num_sms, cudaStream_t stream)
{
    // CTAs of a row: as many as find room at once, none for less than a batch
    const long long items = (long long)p.B * p.n;
    const int batch = kLogThreads * kLogLoads * (p.bf16 ? 8 : 4);
    p.cluster = 1;
    while (p.cluster < kMaxCluster && items * p.cluster * 2 <= 4ll * num_sms && p.V > p.cluster * batch) p.cluster *= 2;
    const dim3 grid((unsigned)(items * p.cluster)), cl((unsigned)p.cluster);
    return p.bf16 ? launch_chained(token_logprobs_kernel<true>, grid, dim3(kLogThreads), cl, stream, p)
                  : launch_chained(token_logprobs_kernel<false>, grid, dim3(kLogThreads), cl, stream, p);
}

}  // namespace ppd
