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
// Bound: instructions, then HBM.  With a key made of every entry and sums one entry at a time, 2048 rows
// of 128,256 bf16 logits took 885 us; 132 now (20 alternatives; 93 without, 77 their bytes alone).
// A batch's maximum propagates NaN and says whether anything of it may be among the best; bf16 entries
// are compared, clamped and maximised two at a time, sums take two fp32 operations an instruction;
// entries are compared with the token as numbers, in columns before it with the next number below it
// (equals rank better there); and no key is made but of what is pushed.  For few rows, the chain of a
// batch: one row of 50,257 takes 9.8 us, 6.4 without alternatives.
//
// The K best: entries that beat the K-th best so far are pushed onto a list, without a barrier; after
// 1, 2, 4, 8, ... batches the list and the best so far are ranked by counting (an entry's place
// is the number of better ones).  As many batches as there were before bring about K that beat the
// K-th best of those, so few are ever pushed.  Where there is no such bound (the first batch), or more
// than fit were pushed (rows that rise: their batches are gone through again), a batch's K-th
// best is bounded from below by the K-th best of the threads' maxima: K threads hold all that are
// better.
#include "ppd_device.cuh"
#include "ppd_kernels.h"

#include <climits>
#include <cmath>
#include <type_traits>

namespace ppd {

constexpr int kLogLoads = 4;                   // 16-byte loads of a batch and thread

// The value behind a rank_key.
PPD_DEV float key_value(uint32_t k)
{
    if (k == 0xFFFFFFFFu) return NAN;
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}

// Running statistics over entries; bad: a NaN or +inf.
struct RowStats {
    float m, s, u;
    int better, bad;
};

// k (x - m).  Half of x and m where k is below 1: their difference may then be past fp32's range
// and its product with k not.
PPD_DEV float exponent(float x, float m, const LogScale &r) { return __fmul_rn(fmaf(x, r.h, -r.h * m), r.kh); }
// The same between two maxima (NaN where both are -inf: -200).
PPD_DEV float exponent_of_max(float a, float m, const LogScale &r) { return fmaxf(exponent(a, m, r), -200.f); }

PPD_DEV void merge_stats(RowStats &a, const RowStats &o, const LogScale &r)
{
    const float nm = fmaxf(a.m, o.m);
    if (nm > -INFINITY) {
        // 2^d (s, u + d s) with d = k (m - nm) <= 0; nothing where there was no entry
        const float da = exponent_of_max(a.m, nm, r), db = exponent_of_max(o.m, nm, r);
        const float wa = a.m > -INFINITY ? ex2(da) : 0.f, wb = o.m > -INFINITY ? ex2(db) : 0.f;
        a.u = wa * fmaf(da, a.s, a.u) + wb * fmaf(db, o.s, o.u);
        a.s = wa * a.s + wb * o.s;
    }
    a.m = nm;
    a.better += o.better;
    a.bad |= o.bad;
}

PPD_DEV __nv_bfloat162 as_bf162(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162 *>(&w); }
PPD_DEV float max3_nan(float a, float b, float c)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// The largest number below x (of the logits' type); NaN below -inf, which nothing is <= to.
template <bool BF16>
PPD_DEV float below(float x)
{
    constexpr uint32_t one = BF16 ? 0x10000u : 1u;
    if (x == 0.f) return __uint_as_float(0x80000000u | one);
    const uint32_t u = __float_as_uint(x);
    if (u == 0xFF800000u) return NAN;
    return __uint_as_float((u & 0x80000000u) ? u + one : u - one);
}

// STAGES: batches on their way or in hand.
template <bool BF16, int THREADS, int STAGES>
__global__ void __launch_bounds__(THREADS) token_logprobs_kernel(const LogprobParams p)
{
    constexpr int E = BF16 ? 8 : 4;            // entries of a load
    constexpr int NV = E * kLogLoads;          // of a batch and thread
    constexpr int WARPS = THREADS / 32;
    constexpr int eb = BF16 ? 2 : 4;
    constexpr uint32_t kAbsent = BF16 ? 0xFF80FF80u : 0xFF800000u;   // -inf
    // An entry of a batch among its others: of bf16 the key's upper half (the lower says nothing) and
    // the column's place from the end, half the instructions of 64 bits.
    using Best = std::conditional_t<BF16, uint32_t, unsigned long long>;
    static_assert(kLogMaxK <= THREADS && kMaxCluster <= NV && kLogLoads * THREADS * E <= 65536, "lists");
    extern __shared__ uint4 s_dyn[];
    auto s_batch = reinterpret_cast<uint4 (*)[kLogLoads][THREADS]>(s_dyn);   // [STAGES]; a thread reads what it asked for itself
    auto s_push = reinterpret_cast<unsigned long long *>(s_batch + STAGES);   // [K NV]: K threads' entries, or a cluster's lists
    __shared__ unsigned long long s_list[2][kLogMaxK], s_bound;
    __shared__ __align__(16) Best s_best[THREADS];
    __shared__ RowStats s_stats[WARPS], s_cta;
    __shared__ int s_n, s_over;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, K = p.K, V = p.V, max_push = K * NV;
    const int rank = (int)blockIdx.x % p.cluster;
    const int item = (int)blockIdx.x / p.cluster;
    const int b = item / p.n, i = item - b * p.n;
    pdl_wait();
    pdl_release();

    // ---- what is asked (the same for the whole cluster)
    auto row_of = [&](int it, int at) { return p.rows ? ld_input(p.rows + it) : at; };
    auto outside = [&](int r, int t) { return r < -1 || r >= p.T || t < -1 || t >= V; };
    auto sequence_status = [&]() {   // by the last CTA of a sequence's first item
        bool any = false;
        for (int x = tid; x < p.n; x += THREADS) any |= outside(row_of(item + x, x), ld_input(p.tokens + item + x));
        any = __syncthreads_or(any);
        if (tid == 0) p.dev_status[b] = any ? kErrTree : kOk;
    };
    const int row = row_of(item, i), token = ld_input(p.tokens + item);
    if (row < 0 || outside(row, token)) {
        if (i == 0 && rank == p.cluster - 1) sequence_status();
        if (rank == 0) {
            if (tid == 0) {
                p.logprob[item] = 0.f;
                p.entropy[item] = 0.f;
                p.rank[item] = -1;
            }
            for (int x = tid; x < K; x += THREADS) {
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
    // ---- groups of E entries on 16 bytes: group g holds columns [g E - skew, ...), groups
    // [f0, f1) of the CTA's [g0, g1) lie inside the row
    const int skew = (int)(reinterpret_cast<uintptr_t>(x0) & 15) / eb;
    const int groups = (int)(((long long)V + skew + E - 1) / E);
    const int g0 = (int)((long long)groups * rank / p.cluster), g1 = (int)((long long)groups * (rank + 1) / p.cluster);
    const int f0 = max(g0, skew ? 1 : 0), f1 = min(g1, (int)(((long long)V + skew) / E));
    const char *xg = x0 - skew * eb;
    constexpr int kStep = kLogLoads * THREADS;
    const int batches = (g1 - g0 + kStep - 1) / kStep;
    // Batch n on its way to its stage (STAGES - 1 batches ahead of the one in hand: 2 KB a warp each).
    auto ask = [&](int n) {
        uint4 *stage = &s_batch[n % STAGES][0][tid];
        const int base = g0 + n * kStep;
        if (base >= f0 && base + kStep <= f1) {
            const char *src = xg + ((size_t)base + tid) * 16;
#pragma unroll
            for (int q = 0; q < kLogLoads; ++q) cp_async16(smem_addr(stage + q * THREADS), src + (size_t)q * THREADS * 16, 16);
        } else if (base < g1) {
#pragma unroll 1
            for (int q = 0; q < kLogLoads; ++q) {
                const int g = base + q * THREADS + tid;
                if (g >= f0 && g < f1) {
                    cp_async16(smem_addr(stage + q * THREADS), xg + (size_t)g * 16, 16);
                    continue;
                }
                // a row's end: the entries that it has
                uint32_t v[4] = {kAbsent, kAbsent, kAbsent, kAbsent};
                const long long c = (long long)g * E - skew;
                if (g < g1) {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        if (c + e < 0 || c + e >= V) continue;
                        const uint32_t y = __float_as_uint(entry_at((int)(c + e)));
                        if (!BF16) v[e & 3] = y;
                        else if (e & 1) v[e / 2] = (v[e / 2] & 0xFFFFu) | y;
                        else v[e / 2] = (v[e / 2] & 0xFFFF0000u) | y >> 16;
                    }
                }
                stage[q * THREADS] = make_uint4(v[0], v[1], v[2], v[3]);
            }
        }
        cp_async_commit();
    };
#pragma unroll 1
    for (int n = 0; n < STAGES - 1; ++n) ask(n);

    const float xt = token >= 0 ? entry_at(token) : 0.f;
    const unsigned long long et = rank_entry(rank_key(xt), token);
    // entries that are not <= this rank before the token: in columns before it, and after it
    const float th0 = token < 0 ? INFINITY : below<BF16>(xt), th1 = token < 0 ? INFINITY : xt;
    const bool odd_token = xt != xt;   // (a NaN is compared as an entry)

    RowStats st{-INFINITY, 0.f, 0.f, 0, 0};
    float x_low = 0.f;             // no entry below it adds to s: 2^-200 of m
    int cur = 0, listed = 0;       // the list in use, its entries
    float least = 0.f;             // the list's last entry, once it has K
    bool full = false;
    if (tid < kLogMaxK) s_list[0][tid] = s_list[1][tid] = 0;
    if (tid == 0) s_n = s_over = 0;

    // The list and the pushed entries together, by the whole block (after a barrier).
    auto rank_pushed = [&]() {
        const int n = s_n;
        for (int y = tid; y < n + listed; y += THREADS) {
            const unsigned long long mine = y < n ? s_push[y] : s_list[cur][y - n];
            int place = 0;
#pragma unroll 8
            for (int z = 0; z < n; ++z) place += s_push[z] > mine;
#pragma unroll 4
            for (int z = 0; z < listed; ++z) place += s_list[cur][z] > mine;
            if (place < K) s_list[cur ^ 1][place] = mine;
        }
        listed = min(K, listed + n);
        __syncthreads();
        if (tid < kLogMaxK) s_list[cur][tid] = 0;   // (for the ranking after the next)
        cur ^= 1;
        const unsigned long long last = s_list[cur][K - 1];
        full = last != 0;
        least = key_value((uint32_t)(last >> 32));
        if (tid == 0) s_n = 0;
        __syncthreads();
    };

    // Rare work (the token's own group, numbers near the type's ends, pushes) is done in rolled
    // loops over what lies in shared memory: the code of a batch is a few hundred instructions,
    // which the instruction cache holds.
    bool bounded = true;           // batch by batch, with a bound of its own
    bool again = false;            // ... of batches whose sums are taken
    int from = 0, to = 1;          // the batches that are ranked together
#pragma unroll 1
    for (int n = 0; n < batches; ++n) {
        ask(n + STAGES - 1);
        cp_async_wait<STAGES - 1>();
        const uint4 *stage = &s_batch[n % STAGES][0][tid];
        const int base = g0 + n * kStep;
        uint4 w[kLogLoads];
#pragma unroll
        for (int q = 0; q < kLogLoads; ++q) w[q] = stage[q * THREADS];
        auto group = [&](int q) { return base + q * THREADS + tid; };
        auto word = [&](const uint4 &r, int x) { return x == 0 ? r.x : x == 1 ? r.y : x == 2 ? r.z : r.w; };
        auto value = [&](const uint4 &r, int e) {   // entry e of a load's E
            if (!BF16) return __uint_as_float(word(r, e));
            return __uint_as_float((e & 1) ? (word(r, e / 2) & 0xFFFF0000u) : (word(r, e / 2) << 16));
        };
        auto column = [&](int q, int e) { return (long long)group(q) * E - skew + e; };
        auto live = [&](int q, int e) { return group(q) < g1 && column(q, e) >= 0 && column(q, e) < V; };

        // ---- the batch's maximum, NaN where there is one
        float mb;
        if (BF16) {
            __nv_bfloat162 a = as_bf162(w[0].x), c = as_bf162(w[0].y);
            a = __hmax2_nan(a, as_bf162(w[0].z)), c = __hmax2_nan(c, as_bf162(w[0].w));
#pragma unroll
            for (int q = 1; q < kLogLoads; ++q) {
                a = __hmax2_nan(__hmax2_nan(a, as_bf162(w[q].x)), as_bf162(w[q].z));
                c = __hmax2_nan(__hmax2_nan(c, as_bf162(w[q].y)), as_bf162(w[q].w));
            }
            a = __hmax2_nan(a, c);
            mb = max3_nan(__low2float(a), __high2float(a), -INFINITY);
        } else {
            float a = -INFINITY, c = -INFINITY;
#pragma unroll
            for (int q = 0; q < kLogLoads; ++q) {
                a = max3_nan(a, value(w[q], 0), value(w[q], 1));
                c = max3_nan(c, value(w[q], E > 2 ? 2 : 0), value(w[q], E > 2 ? 3 : 1));
            }
            mb = max3_nan(a, c, -INFINITY);
        }
        if (!again) {
            st.bad |= !(mb < INFINITY);
            if (mb > st.m) {
                const float d = exponent_of_max(st.m, mb, p.scale), f = ex2(d);   // (s is 0 where m was -inf)
                st.u = f * fmaf(d, st.s, st.u);
                st.s *= f;
                st.m = mb;
                x_low = __fsub_rd(mb, p.scale.span);
            }
            // ---- sums
            const bool far = __any_sync(0xffffffffu, mb > -INFINITY && !(fabsf(st.m) < p.scale.fused));   // (a warp together)
            if (mb == -INFINITY) {
                // nothing to add
            } else if (!far) {
                // x k - M in one operation; M, m k rounded, is off by 2^-5 at most, which sums are
                // freed of after the batch (from |m k| = 2^31 on 2 to that could be past fp32's range)
                const float nm = -__fmul_rn(st.m, p.scale.k);
                const uint64_t nm2 = pack2(nm, nm), k2 = pack2(p.scale.k, p.scale.k);
                uint64_t s2 = 0ull, u2 = 0ull;
                const __nv_bfloat162 low2 = __bfloat162bfloat162(__float2bfloat16_rd(x_low));
#pragma unroll
                for (int q = 0; q < kLogLoads; ++q) {
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        float a, c;
                        if (BF16) {
                            const __nv_bfloat162 v = __hmax2(as_bf162(word(w[q], e / 2)), low2);
                            const uint32_t x = *reinterpret_cast<const uint32_t *>(&v);
                            a = __uint_as_float(x << 16), c = __uint_as_float(x & 0xFFFF0000u);
                        } else {
                            a = fmaxf(value(w[q], e), x_low), c = fmaxf(value(w[q], e + 1), x_low);
                        }
                        const uint64_t d2 = fma2(pack2(a, c), k2, nm2);
                        unpack2(d2, a, c);
                        const uint64_t v2 = pack2(ex2(a), ex2(c));
                        s2 = add2(s2, v2);
                        u2 = fma2(v2, d2, u2);
                    }
                }
                float a, c, e, g;
                unpack2(s2, a, c);
                unpack2(u2, e, g);
                const float off = fmaf(st.m, p.scale.k, nm), f = ex2(-off), s = a + c;
                st.s = fmaf(f, s, st.s);
                st.u = fmaf(f, fmaf(-off, s, e + g), st.u);
            } else {
                // far from 0: x - m first; exponents clamped, not entries (2048 rows of 128,256 bf16, all but a
                // ten-thousandth masked with -1e9, 152 us; with -1e4 136)
                const float nm = -p.scale.h * st.m;
                uint64_t s2 = 0ull, u2 = 0ull;
#pragma unroll 1
                for (int q = 0; q < kLogLoads; ++q) {
                    const uint4 r = stage[q * THREADS];
#pragma unroll
                    for (int e = 0; e < E; e += 2) {
                        float a, c;
                        unpack2(mul2(fma2(pack2(value(r, e), value(r, e + 1)), pack2(p.scale.h, p.scale.h), pack2(nm, nm)), pack2(p.scale.kh, p.scale.kh)), a, c);
                        a = fmaxf(a, -200.f), c = fmaxf(c, -200.f);   // (2^-200 is 0; nothing times an infinity)
                        const uint64_t v2 = pack2(ex2(a), ex2(c));
                        s2 = add2(s2, v2);
                        u2 = fma2(v2, pack2(a, c), u2);
                    }
                }
                float a, c;
                unpack2(s2, a, c);
                st.s += a + c;
                unpack2(u2, a, c);
                st.u += a + c;
            }
            // ---- entries that rank before the token
            const long long c0 = (long long)base * E - skew;   // the batch's first column
            if (base >= f0 && base + kStep <= f1 && !odd_token && (token < c0 || token >= c0 + (long long)kStep * E)) {
                const float th = c0 < token ? th0 : th1;
                if (BF16) {
                    const __nv_bfloat162 th2 = __bfloat162bfloat162(__float2bfloat16_rn(th));
                    __nv_bfloat162 n2 = __hgtu2(as_bf162(w[0].x), th2);
#pragma unroll
                    for (int x = 1; x < 4 * kLogLoads; ++x) n2 = __hadd2(n2, __hgtu2(as_bf162(word(w[x / 4], x % 4)), th2));
                    st.better += (int)(__low2float(n2) + __high2float(n2));
                } else {
#pragma unroll
                    for (int q = 0; q < kLogLoads; ++q)
#pragma unroll
                        for (int e = 0; e < E; ++e) st.better += !(value(w[q], e) <= th);
                }
            } else {   // the batch of the token, or a row's end: the loads that hold them entry by entry
#pragma unroll 1
                for (int q = 0; q < kLogLoads; ++q) {
                    const uint4 r = stage[q * THREADS];
                    const int g = group(q);
                    const long long c = column(q, 0);
                    if (g >= g1) continue;
                    if (odd_token || (c <= token && token < c + E) || g < f0 || g >= f1) {
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            st.better += live(q, e) && rank_entry(rank_key(value(r, e)), (int)c + e) > et;
                    } else {
                        const float th = c < token ? th0 : th1;
#pragma unroll
                        for (int e = 0; e < E; ++e) st.better += !(value(r, e) <= th);
                    }
                }
            }
        }
        if (K == 0) continue;

        // ---- the K best
        // one bit for each of a thread's entries: of bf16, bit x the low half of word x, bit 16 + x the high one
        auto bits = [&](auto test2, auto test) {
            uint32_t some = 0;
#pragma unroll
            for (int q = 0; q < kLogLoads; ++q)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if (BF16) some |= test2(as_bf162(word(w[q], x))) & 0x10001u << (4 * q + x);
                    else some |= (test(value(w[q], x)) ? 1u : 0u) << (4 * q + x);
                }
            return some;
        };
        auto in_order = [](int bit) { return BF16 ? 2 * (bit & 15) + (bit >> 4) : bit; };
        auto stored = [&](int at) {   // entry `at` in order
            const uint32_t y = reinterpret_cast<const uint32_t *>(stage + at / E * THREADS)[BF16 ? at % E / 2 : at % E];
            return __uint_as_float(!BF16 ? y : (at & 1) ? (y & 0xFFFF0000u) : y << 16);
        };
        const bool sees = full ? !(mb <= least) && least == least : group(0) < g1;
        const bool plain = full && !bounded;
        // entries that are not <= t are pushed: all that beat the list (equal ones come later), or
        // those of at least `bound`
        float t = least;
        unsigned long long bound = 0;
        if (!plain) {
            bound = full ? (unsigned long long)(rank_key(least) + 1) << 32 : 1;
            if (bounded) {
                // this thread's best entry: the first of the batch's largest
                Best gm = 0;
                int at = 0;
                if (sees) {
                    if (mb > -INFINITY) {
                        const __nv_bfloat162 mb2 = __bfloat162bfloat162(__float2bfloat16_rn(mb));
                        const uint32_t same = bits([&](__nv_bfloat162 v) { return __heq2_mask(v, mb2); }, [&](float v) { return v == mb; });
                        at = in_order(__ffs(same) - 1);
                        if (BF16 && (same & 0xFFFFu) && same >> 16) at = min(in_order(__ffs(same & 0xFFFFu) - 1), in_order(__ffs(same >> 16) + 15));
                    } else if (mb != mb) {
                        while (stored(at) == stored(at)) ++at;
                    } else {   // only -inf: the first entry that there is
                        while (at < NV && !live(at / E, at % E)) ++at;
                    }
                    if (at < NV) {
                        if constexpr (BF16) gm = (rank_key(mb) & 0xFFFF0000u) | (0xFFFFu - (at / E * THREADS + tid) * E - at % E);
                        else gm = rank_entry(rank_key(mb), (int)column(at / E, at % E));
                    }
                }
                s_best[tid] = gm;
                if (tid == 0) s_bound = 0;
                __syncthreads();
                int place = 0;
#pragma unroll 8
                for (int y = 0; y < THREADS; y += 16 / (int)sizeof(Best)) {
                    if constexpr (BF16) {
                        const uint4 z = *reinterpret_cast<const uint4 *>(s_best + y);
                        place += (z.x > gm) + (z.y > gm) + (z.z > gm) + (z.w > gm);
                    } else {
                        const ulonglong2 z = *reinterpret_cast<const ulonglong2 *>(s_best + y);
                        place += (z.x > gm) + (z.y > gm);
                    }
                }
                if (gm != 0 && place == K - 1)   // (fewer than K threads: no bound)
                    s_bound = rank_entry(rank_key(mb), (int)column(at / E, at % E));
                __syncthreads();
                bound = s_bound > bound ? s_bound : bound;
            }
            t = bound > 1 ? below<false>(key_value((uint32_t)(bound >> 32))) : NAN;
        }
        if (sees && !(mb <= t)) {
            const __nv_bfloat162 t2 = __bfloat162bfloat162(__float2bfloat16_rd(t));
            uint32_t some = bits([&](__nv_bfloat162 v) { return __hgtu2_mask(v, t2); }, [&](float v) { return !(v <= t); });
            while (some) {   // (few threads have more than one or two)
                const int at = in_order(__ffs(some) - 1);
                some &= some - 1;
                const unsigned long long en = rank_entry(rank_key(stored(at)), (int)column(at / E, at % E));
                if (!plain && (en < bound || !live(at / E, at % E))) continue;
                const int place = atomicAdd(&s_n, 1);
                if (place < max_push) s_push[place] = en;
                else s_over = 1;   // (not where the batch has a bound)
            }
        }
        if (bounded || n + 1 >= to || n + 1 == batches) {
            __syncthreads();
            if (s_over) {
                // more than fit: the same batches again, one by one
                __syncthreads();
                if (tid == 0) s_n = s_over = 0;   // (barriers before the next push)
                to = min(to, n + 1);
                bounded = again = true;
                cp_async_wait<0>();
#pragma unroll 1
                for (int x = 0; x < STAGES - 1; ++x) ask(from + x);
                n = from - 1;
                continue;
            }
            rank_pushed();
            if (n + 1 >= to) {
                from = n + 1;
                to = 2 * from;
                bounded = again = false;
            }
        }
    }

    // ---- the CTA's statistics, then the cluster's
    auto merge_lanes = [&](int most) {
#pragma unroll 1
        for (int o = most; o > 0; o >>= 1) {
            RowStats y;
            y.m = __shfl_xor_sync(0xffffffffu, st.m, o);
            y.s = __shfl_xor_sync(0xffffffffu, st.s, o);
            y.u = __shfl_xor_sync(0xffffffffu, st.u, o);
            y.better = __shfl_xor_sync(0xffffffffu, st.better, o);
            y.bad = __shfl_xor_sync(0xffffffffu, st.bad, o);
            merge_stats(st, y, p.scale);
        }
    };
    const RowStats empty{-INFINITY, 0.f, 0.f, 0, 0};
    merge_lanes(16);
    if (lane == 0) s_stats[warp] = st;
    if (cur == 1 && tid < K) s_list[0][tid] = s_list[1][tid];
    __syncthreads();
    if (warp == 0) {
        st = lane < WARPS ? s_stats[lane] : empty;
        merge_lanes(WARPS / 2);
        if (lane == 0) s_cta = st;
    }
    if (p.cluster > 1) cluster_sync();
    else __syncthreads();
    if (i == 0 && rank == p.cluster - 1) sequence_status();
    if (rank == 0) {
        // every warp the whole row's statistics
        st = empty;
        if (lane < p.cluster) {
            const uint32_t a = cluster_map(smem_addr(&s_cta), lane);
            st.m = ld_cluster_f32(a);
            st.s = ld_cluster_f32(a + 4);
            st.u = ld_cluster_f32(a + 8);
            st.better = __float_as_int(ld_cluster_f32(a + 12));
            st.bad = __float_as_int(ld_cluster_f32(a + 16));
        }
        merge_lanes(kMaxCluster / 2);   // lane 0's (lanes 0 to 7 agree)
        st.m = __shfl_sync(0xffffffffu, st.m, 0);
        st.s = __shfl_sync(0xffffffffu, st.s, 0);
        st.u = __shfl_sync(0xffffffffu, st.u, 0);
        st.better = __shfl_sync(0xffffffffu, st.better, 0);
        st.bad = __shfl_sync(0xffffffffu, st.bad, 0);
        const bool bad = st.bad || st.m == -INFINITY;
        const float lg = lg2(st.s), ln2 = 0.69314718055994530942f;
        auto logprob = [&](float x) { return bad ? NAN : (exponent(x, st.m, p.scale) - lg) * ln2; };
        if (tid == 0) {
            p.logprob[item] = token < 0 ? 0.f : logprob(xt);
            p.entropy[item] = bad ? NAN : (lg - st.u / st.s) * ln2;
            p.rank[item] = token < 0 ? -1 : st.better;
        }
        // the CTAs' lists together: an entry's place is the number of better ones
        const int n = p.cluster * K;
        for (int y = tid; y < n; y += THREADS)
            s_push[y] = y < K ? s_list[0][y] : ld_cluster_u64(cluster_map(smem_addr(&s_list[0][0]) + (uint32_t)(y % K) * 8, y / K));
        __syncthreads();
        for (int y = tid; y < n; y += THREADS) {
            const unsigned long long mine = s_push[y];
            int place = 0;
#pragma unroll 8
            for (int z = 0; z < n; ++z) place += s_push[z] > mine;
            if (mine != 0 && place < K) {
                p.top_tokens[(size_t)item * K + place] = entry_index(mine);
                p.top_logprobs[(size_t)item * K + place] = logprob(key_value((uint32_t)(mine >> 32)));
            }
        }
    }
    if (p.cluster > 1) cluster_sync();   // no list that a peer reads goes away
}

// Threads of a block where rows are many: with fewer, barriers cost less and as many rows as there are find
// room at once (an SM takes 8, 16 or 32 blocks, by registers), but a warp has more of a long row and of a
// ranking to itself.  128 / 64 / 32, us:
//   rows                 of           alternatives: 5               20                   32
//   14,400 (95 an SM)    1000 fp32    121 /  65 /  42       128 /  71 /  56      134 /  76 / 108
//   6000 (39)            32,000 bf16  136 / 112 /  99       154 / 133 / 131      166 / 157 / 204
//   4000 (26)            16,000 bf16   69 /  54 /  47        77 /  64 /  68       83 /  80 / 108
//   3000 (20)            32,000 bf16   72 /  62 /  69        81 /  74 /  76       88 /  88 / 147
//   2000 (13)            32,000 bf16   50 /  46 /  44        57 /  54 /  70       62 /  70 /  87
//   1500 (10)            32,000 bf16   40 /  43 /  38        46 /  50 /  51       50 /  51 /  84
//   1400 (9)             4000 bf16     17 /  16 /  13        19 /  18 /  17       19 /  18 /  41
//   4000 (26)            128,256 bf16 212 / 205 / 222       239 / 234 / 265      258 / 270 / 319
//   2048 (13)            128,256 bf16 117 / 123 / 129       132 / 136 / 187      142 / 166 / 189
static int log_threads(long long rows_a_sm, int K, long long row_bytes)
{
    if (K <= 20 && (row_bytes <= 8192 || (rows_a_sm >= 32 && row_bytes <= 65536))) return 32;
    if (rows_a_sm >= 16 || (rows_a_sm >= 12 && K <= 20 && row_bytes <= 131072)) return 64;
    return 128;
}

cudaError_t launch_token_logprobs(LogprobParams p, int num_sms, cudaStream_t stream)
{
    // CTAs of a row: as many as are all resident at once with four stages (five an SM), none for
    // less than a batch.  1 / 2 / 4 / 8 of them, us, 20 alternatives:
    //   150 rows of 128,256 fp32   47 / 34 / 33 / 43        320 of 256,000 bf16    67 / 58 / 64 / 80
    //   16 rows of 128,256 fp32    47 / 31 / 22 / 19        2000 of 32,000 bf16    59 / 78 / 115 / 210
    // Four stages, 33 to 43 KB, where no more than those run (700 rows of 256,000 bf16: 93 us, with two
    // stages 122); else two, so that eight CTAs find room (2048 rows of 128,256 bf16: 133 us, with
    // four 162), or more of fewer threads.
    const long long items = (long long)p.B * p.n;
    const int batch = 128 * kLogLoads * (p.bf16 ? 8 : 4);
    p.cluster = 1;
    while (p.cluster < kMaxCluster && items * p.cluster * 2 <= 5ll * num_sms && p.V > p.cluster * batch) p.cluster *= 2;
    const bool deep = items * p.cluster <= 5ll * num_sms;
    const int threads = deep ? 128 : log_threads(items / num_sms, p.K, (long long)p.V * (p.bf16 ? 2 : 4));
    auto launch = [&](auto kern, int stages) {
        const uint32_t smem = (uint32_t)(stages * kLogLoads * threads * 16 + p.K * kLogLoads * (p.bf16 ? 8 : 4) * 8);
        return launch_chained_smem(kern, dim3((unsigned)(items * p.cluster)), dim3((unsigned)threads), dim3((unsigned)p.cluster), smem, stream, p);
    };
    if (deep) return p.bf16 ? launch(token_logprobs_kernel<true, 128, 4>, 4) : launch(token_logprobs_kernel<false, 128, 4>, 4);
    if (threads == 128) return p.bf16 ? launch(token_logprobs_kernel<true, 128, 2>, 2) : launch(token_logprobs_kernel<false, 128, 2>, 2);
    if (threads == 64) return p.bf16 ? launch(token_logprobs_kernel<true, 64, 2>, 2) : launch(token_logprobs_kernel<false, 64, 2>, 2);
    return p.bf16 ? launch(token_logprobs_kernel<true, 32, 2>, 2) : launch(token_logprobs_kernel<false, 32, 2>, 2);
}

}  // namespace ppd
