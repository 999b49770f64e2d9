// ppd_kv4.cu -- the 4-bit cache: rows into it (ppd_kv4_append), back out (ppd_kv4_read),
// and the tree's attention over it for few query rows (single tokens, small trees).
#include "ppd_kv4.cuh"

#include <cmath>

namespace ppd {

// ------------------------------------------------------------------ rows in

// Eight channels of a source row as fp32.
PPD_DEV void ld_eight(const void *p, size_t i, bool f32, float (&v)[8])
{
    if (f32) {
        const float4 *f = reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(p) + i);
        const float4 a = ld_input(f), b = ld_input(f + 1);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        return;
    }
    const uint4 a = ld_input(reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(p) + i));
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) v[2 * e] = __uint_as_float(w[e] << 16), v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
}

// A sequence's rows are refused as a whole: a start or a count outside the cache.
PPD_DEV int append_status(int start, int n, int T, int S_max)
{
    return start < 0 || n < 0 || n > T || start > S_max || n > S_max - start ? kErrCapacity : kOk;
}

// A block takes kAppendRows new rows of a slice, K and V.  A thread quantises the eight channels
// of one word of codes, four threads share a scale: the largest magnitude by two shuffles, then
// two roundings alone: a / 7 (then up to the next scale) and x / s.  The quotient is x times
// the rounded reciprocal with one Newton step, which rounds it correctly (Markstein's theorem:
// an fp32 reciprocal rounded to nearest, and a fused residual); halves are then exact, and
// adding 1.5 * 2^23 + 8 rounds to the nearest integer, half to even, and leaves the code in the low
// bits.  Divisions in their place were 43 of a prompt's 67 us.  Four rows' loads a thread in flight.
// Bound by instruction issue, then by HBM: 256 slices of 1003 fp32 rows into the cache and out of it
// (D = 64, 232 MB) 56 us, 4.2 TB/s.
constexpr int kAppendRows = 64, kAppendDeep = 4;
template <int D>
__global__ void __launch_bounds__(256) kv4_append_kernel(const Kv4AppendParams p)
{
    pdl_release();
    pdl_wait();
    constexpr int LANES = D / 8;
    const int lane = threadIdx.x % LANES, first = threadIdx.x / LANES;
    constexpr int STEP = 256 / LANES;   // (row, K or V) pairs of a pass
    const long long u = blockIdx.x;
    const int b = (int)(u / p.H % p.B);
    const int start = ld_input(p.start + b), n = ld_input(p.n_new + b);
    const int status = append_status(start, n, p.T, p.S_max);
    if (u / p.H < p.B && u % p.H == 0 && blockIdx.y == 0 && threadIdx.x == 0) p.dev_status[b] = status;
    if (status != kOk) return;
    const int j0 = (int)blockIdx.y * kAppendRows, pairs = 2 * (min(n, j0 + kAppendRows) - j0);
    for (int i0 = 0; i0 < pairs; i0 += kAppendDeep * STEP) {   // the same for every thread: shuffles follow
        float v[kAppendDeep][8];
        bool real[kAppendDeep];
#pragma unroll
        for (int k = 0; k < kAppendDeep; ++k) {
            const int i = i0 + k * STEP + first, j = j0 + (i >> 1);
            int src = i < pairs ? j : -1;
            if (src >= 0 && p.rows) src = ld_input(p.rows + (size_t)b * p.T + j);
            real[k] = src >= 0 && src < p.T;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] = 0.f;
            if (real[k]) ld_eight(i & 1 ? p.v_new : p.k_new, ((size_t)u * p.T + src) * D + 8 * lane, p.f32, v[k]);
        }
#pragma unroll
        for (int k = 0; k < kAppendDeep; ++k) {
            if (i0 + k * STEP >= pairs) break;
            float a = 0.f;   // fmaxf passes a NaN by
#pragma unroll
            for (int e = 0; e < 8; ++e) a = fmaxf(a, fabsf(v[k][e]));
            a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));
            a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 2));
            const int up = (int)((__float_as_uint(__fdiv_rn(a, 7.f)) + 0xFFFFFu) >> 20) - 107 * 8;
            const uint32_t sb = (uint32_t)min(max(up, 0), 255);
            const float s = kv4_scale(sb), top = 7.f * s, inv = __frcp_rn(s);   // (7 s is exact)
            uint32_t word = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = v[k][e] == v[k][e] ? fminf(fmaxf(v[k][e], -top), top) : 0.f;
                const float t = x * inv;
                const uint32_t c = __float_as_uint(fmaf(fmaf(-t, s, x), inv, t) + 12582920.f) & 15u;
                word |= c << (4 * (e >> 1) + 16 * (e & 1));   // even channels in the low half, odd ones in the high half
            }
            const int i = i0 + k * STEP + first;
            if (real[k]) {
                const size_t row = (size_t)u * p.S_max + start + j0 + (i >> 1);
                reinterpret_cast<uint32_t *>(i & 1 ? p.v_cache : p.k_cache)[row * LANES + lane] = word;
                if (!(lane & 3)) (i & 1 ? p.v_scale : p.k_scale)[row * (D / kKv4Group) + lane / 4] = (uint8_t)sb;
            }
        }
    }
}

cudaError_t launch_kv4_append(const Kv4AppendParams &p, cudaStream_t stream)
{
    const dim3 grid((unsigned)p.slices, (unsigned)((p.T + kAppendRows - 1) / kAppendRows));
    return p.D == 128 ? launch_chained(kv4_append_kernel<128>, grid, dim3(256), dim3(1), stream, p)
                      : launch_chained(kv4_append_kernel<64>, grid, dim3(256), dim3(1), stream, p);
}

// ------------------------------------------------------------------ rows out

// A thread a word of codes, all slices' rows end to end; four words a thread in flight.
constexpr int kReadDeep = 4;
template <int D>
__global__ void __launch_bounds__(256) kv4_read_kernel(const Kv4ReadParams p)
{
    pdl_release();
    pdl_wait();
    constexpr int WORDS = D / 8;
    const uint32_t rows = (uint32_t)(p.slices * p.N);   // below 2^31
    const int w = threadIdx.x % WORDS;
    const uint32_t row0 = blockIdx.x * (kReadDeep * 256 / WORDS) + threadIdx.x / WORDS;
    uint32_t c[kReadDeep], sb[kReadDeep];
#pragma unroll
    for (int k = 0; k < kReadDeep; ++k) {
        const uint32_t r = row0 + k * (256 / WORDS);
        c[k] = 0x88888888u;   // zeros
        sb[k] = 0;
        if (r >= rows) continue;
        const uint32_t u = r / (uint32_t)p.N;
        const int b = (int)(u / (uint32_t)p.H % (uint32_t)p.B), j = (int)(r - u * p.N);
        const int start = ld_input(p.start + b), n = ld_input(p.n + b);
        if (j < n && start >= 0 && start <= p.S_max && j < p.S_max - start) {
            const size_t row = (size_t)u * p.S_max + start + j;
            c[k] = (uint32_t)ld_input(reinterpret_cast<const int *>(p.cache) + row * WORDS + w);
            asm volatile("ld.global.u8 %0, [%1];" : "=r"(sb[k]) : "l"(p.scale + row * (D / kKv4Group) + w / 4) : "memory");
        }
    }
#pragma unroll
    for (int k = 0; k < kReadDeep; ++k) {
        const uint32_t r = row0 + k * (256 / WORDS);
        if (r >= rows) return;
        uint32_t v[4];
        kv4_word(c[k], kv4_scales(sb[k] * 0x10001u), v);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = kv4_whole(v[e]);
        const size_t at = (size_t)r * D + 8 * w;
        if (!p.f32) {
            *reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(p.out) + at) = make_uint4(v[0], v[1], v[2], v[3]);
        } else {
            float *o = reinterpret_cast<float *>(p.out) + at;
#pragma unroll
            for (int e = 0; e < 4; e += 2)
                *reinterpret_cast<float4 *>(o + 2 * e) =
                    make_float4(__uint_as_float(v[e] << 16), __uint_as_float(v[e] & 0xFFFF0000u),
                                __uint_as_float(v[e + 1] << 16), __uint_as_float(v[e + 1] & 0xFFFF0000u));
        }
    }
}

cudaError_t launch_kv4_read(const Kv4ReadParams &p, cudaStream_t stream)
{
    const long long per = kReadDeep * 256 / (p.D / 8), rows = p.slices * p.N;
    const dim3 grid((unsigned)((rows + per - 1) / per));
    return p.D == 128 ? launch_chained(kv4_read_kernel<128>, grid, dim3(256), dim3(1), stream, p)
                      : launch_chained(kv4_read_kernel<64>, grid, dim3(256), dim3(1), stream, p);
}

// ------------------------------------------------------------------ attention, few rows

// Up to eight query rows of a slice (the G query heads of a K/V head times the T tree tokens; NB = 2
// blocks of eight where D = 64) against a range of its keys, in registers: four warps take chunks
// of 32 keys in turn.  Keys and channels fill the products' 16 rows, queries their eight columns:
//
//   S^T = K Q^T      K's fragments made from the codes a thread loads: thread t of a quad holds
//                    channels [t D / 4, (t + 1) D / 4) of two keys, the order of the channels in
//                    the sum being free as long as Q follows it
//   O^T += V^T P^T   P^T's fragments are S^T's accumulators, transposed in 8 x 8 tiles by
//                    movmatrix; V^T's are made from the codes of two neighbouring keys at once,
//                    thread g of a column holding channels [g D / 8, (g + 1) D / 8)
//
// with a running reference kKv4Shift below the maximum (what takes the values' unit up again),
// which moves when a score passes the maximum by 2^8, and P as bf16 hi + lo
// (2^-18: V's values are exact, so the output's own rounding is all that shows).  Each warp's
// state is merged in shared memory, those of a split slice by kv4_merge_kernel.  A chunk's
// codes and scales come by asynchronous copies into a ring of the warp's own: no barrier in the
// loop.
//
// Bound by the latency of a warp's chain from codes to products, which four blocks an SM do not
// hide: issue slots are 56 % used, the tensor pipe 29 %, and a warp waits most for results of fixed
// latency (some 735 instructions for a chunk of 32 keys, D = 128); 64 x 32 slices of 2048 keys 163 us,
// 3.5 TB/s.  Few slices are bound by a block's start and end and by the merge (issue 41 %): 32 slices
// of 10,000 keys 20.4 to 21.5 us, 1.7 TB/s.
template <int D>
struct Kv4Few {
    static constexpr int WARPS = 4, THREADS = 128, KEYS = 32;
    static constexpr int STAGES = 3;
    static constexpr int RB = D / 2;                         // bytes of a row's codes
    static constexpr int SB = D / kKv4Group;                 // scale bytes of a row
    static constexpr uint32_t CODES = KEYS * RB;             // of K, or V, in a stage
    static constexpr uint32_t OFF_SC = 2 * CODES;            // scales, a word a key: K's, then V's
    static constexpr uint32_t STAGE = 2 * CODES + 2 * KEYS * 4;
    static constexpr uint32_t RING = WARPS * STAGES * STAGE; // merge: [WARPS][rows][D] over the ring
    static constexpr uint32_t OFF_ML = RING;                 // [WARPS][16]: reference, sum
    static constexpr uint32_t OFF_PARENT = OFF_ML + WARPS * 16 * 8;
    static constexpr uint32_t SMEM = OFF_PARENT + kMaxTree * 4;
    static_assert(WARPS * 16 * D * 4 <= RING, "the states fit over the ring");
};

template <int D, int NB>
__global__ void __launch_bounds__(Kv4Few<D>::THREADS, NB == 1 ? 4 : 3) kv4_attention_few_kernel(const Kv4AttnParams p)
{
    using C = Kv4Few<D>;
    extern __shared__ __align__(16) uint8_t smem[];
    pdl_release();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int split = (int)(blockIdx.x % p.splits);
    const uint32_t u = blockIdx.x / p.splits;
    const int b = (int)(u / (uint32_t)p.H % (uint32_t)p.B);
    const int T = p.T, R = p.G * T;
    const int32_t *parent = p.parent + (size_t)b * T;
    const int P_in = ld_input(p.prefix_len + b);
    const int P = min(max(P_in, 0), p.S_max);
    if (u % p.H == 0 && u / p.H < p.B && split == 0 && warp == 0) {
        const int st = tree_status(parent, T, P_in, p.S_max, lane);
        if (lane == 0) p.dev_status[b] = st;
    }
    const int n_pref = (P + C::KEYS - 1) / C::KEYS, n_all = n_pref + (T + C::KEYS - 1) / C::KEYS;
    const int c0 = (int)((long long)n_all * split / p.splits), c1 = (int)((long long)n_all * (split + 1) / p.splits);

    int *par = reinterpret_cast<int *>(smem + C::OFF_PARENT);
    if (c1 > n_pref) {   // this part has tree keys: their rows are read when their turn comes
        for (int i = threadIdx.x; i < T; i += C::THREADS) par[i] = ld_input(parent + i);
        const size_t bytes = (size_t)T * D * (p.f32 ? 4 : 2);
        for (size_t i = (size_t)threadIdx.x * 128; i < bytes; i += C::THREADS * 128) {
            asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const uint8_t *>(p.k_tree) + u * bytes + i));
            asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const uint8_t *>(p.v_tree) + u * bytes + i));
        }
    }

    const uint32_t ring = smem_addr(smem) + warp * C::STAGES * C::STAGE;
    const size_t row0 = (size_t)u * p.S_max;
    // Where the warp's loads of V take a row's 16-byte pieces: rows 2t of a column's threads
    // (2t + 1 likewise) lie in different banks.
    auto v_swizzle = [](int row) {
        return D == 128 ? (((row >> 1) & 1) << 1) | (((row >> 2) & 1) << 2) : ((row >> 2) & 1) << 1;
    };
    constexpr int UPR = C::RB / 16;   // 16-byte pieces of a row; piece i of a lane is 512 bytes on from piece i - 1
    const uint32_t to_v = (uint32_t)(lane ^ v_swizzle(lane / UPR)) * 16;   // (the swizzle repeats every 512 bytes)
    auto fetch = [&](int c, int stage) {
        if (c < min(c1, n_pref)) {
            const int k0 = c * C::KEYS, n = P - k0;
            const uint32_t dst = ring + stage * C::STAGE;
            const size_t at = (row0 + k0) * C::RB + lane * 16;
            const uint8_t *k = p.k_cache + at, *v = p.v_cache + at;
            if (D == 128 && n >= C::KEYS) {
                const size_t a = (row0 + k0 + lane) * C::SB;
#pragma unroll
                for (int i = 0; i < UPR; ++i) {
                    cp_async16(dst + lane * 16 + i * 512, k + i * 512, 16u);
                    cp_async16(dst + C::CODES + to_v + i * 512, v + i * 512, 16u);
                }
                cp_async4(dst + C::OFF_SC + lane * 4, p.k_scale + a, 4u);
                cp_async4(dst + C::OFF_SC + 128 + lane * 4, p.v_scale + a, 4u);
            } else {
#pragma unroll
                for (int i = 0; i < UPR; ++i) {
                    const bool in = i * (32 / UPR) + lane / UPR < n;   // rows past the prefix arrive as zeros (finite: scale 2^-20)
                    cp_async16(dst + lane * 16 + i * 512, in ? k + i * 512 : p.k_cache, in ? 16u : 0u);
                    cp_async16(dst + C::CODES + to_v + i * 512, in ? v + i * 512 : p.v_cache, in ? 16u : 0u);
                }
                // a word holds the row's scales (D = 64: those of an even and an odd row; the
                // tensors' last word may be half one)
                const bool in = lane < n;
                const size_t a = ((row0 + (in ? k0 + lane : 0)) * C::SB) & ~(size_t)3;
                const size_t left = p.scale_bytes - a;
                const uint32_t m = in ? (left < 4 ? (uint32_t)left : 4u) : 0u;
                cp_async4(dst + C::OFF_SC + lane * 4, p.k_scale + a, m);
                cp_async4(dst + C::OFF_SC + 128 + lane * 4, p.v_scale + a, m);
            }
        }
        cp_async_commit();
    };
    int next = c0 + warp;   // the next chunk to fetch
#pragma unroll
    for (int s = 0; s < C::STAGES - 1; ++s, next += C::WARPS) fetch(next, s);

    // Q's fragments: rows g of the blocks
    const size_t q_row0 = (size_t)u * R;
    uint32_t q[NB][D / 16][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int r = 8 * nb + g;
        const size_t at = (q_row0 + (r < R ? r : 0)) * D + (D / 4) * t;
        if (!p.f32) {
            const uint4 *src = reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(p.q) + at);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                const uint4 v = r < R ? ld_input(src + i) : make_uint4(0, 0, 0, 0);
                q[nb][2 * i][0] = v.x, q[nb][2 * i][1] = v.y, q[nb][2 * i + 1][0] = v.z, q[nb][2 * i + 1][1] = v.w;
            }
        } else {
            const float4 *src = reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(p.q) + at);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const float4 v = r < R ? ld_input(src + i) : make_float4(0.f, 0.f, 0.f, 0.f);
                q[nb][i][0] = bf16x2(v.x, v.y), q[nb][i][1] = bf16x2(v.z, v.w);
            }
        }
    }
    float o[D / 16][NB][4] = {};   // kKv4Unit times the sums: channels g D / 8 + i and D / 16 on, queries 2t and 2t + 1
    float m[NB][2], l[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) m[nb][0] = m[nb][1] = -INFINITY, l[nb][0] = l[nb][1] = 0.f;
    __syncthreads();   // the parents are in shared memory

    int stage = 0;
    for (int c = c0 + warp; c < c1; c += C::WARPS) {
        fetch(next, stage == 0 ? C::STAGES - 1 : stage - 1);
        next += C::WARPS;
        cp_async_wait<C::STAGES - 1>();
        __syncwarp();
        const bool tree = c >= n_pref;
        const int k0 = (tree ? c - n_pref : c) * C::KEYS;
        const uint32_t src = ring + stage * C::STAGE;
        const uint32_t odd = D == 64 ? (uint32_t)(row0 + k0) & 1u : 0u;   // which half of a word is row 0's
        float s[2][NB][4] = {};
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            if (!tree) {
                uint32_t w[2][D / 32];
                Kv4Scale sc[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t row = 16 * mt + 8 * h + g;
                    if constexpr (D == 128) {
                        const uint4 v = ld_shared_u128(src + row * 64u + t * 16u);
                        w[h][0] = v.x, w[h][1] = v.y, w[h][2] = v.z, w[h][3] = v.w;
                    } else {
                        const uint2 v = ld_shared_u64(src + row * 32u + t * 8u);
                        w[h][0] = v.x, w[h][1] = v.y;
                    }
                    const uint32_t at = D == 128 ? t : (((row ^ odd) & 1u) << 1) + (t >> 1);
                    sc[h] = kv4_scales(ld_shared_u8(src + C::OFF_SC + row * 4u + at) * 0x10001u);
                }
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t x0 = w[0][k >> 1] >> (8 * (k & 1)), x1 = w[1][k >> 1] >> (8 * (k & 1));
                    const uint32_t a[4] = {kv4_low(x0, sc[0]), kv4_low(x1, sc[1]), kv4_high(x0, sc[0]), kv4_high(x1, sc[1])};
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) mma_bf16(s[mt][nb], a, q[nb][k][0], q[nb][k][1]);
                }
            } else {
                const int j0 = k0 + 16 * mt + g, j1 = j0 + 8;
                const size_t at0 = ((size_t)u * T + (j0 < T ? j0 : 0)) * D + (D / 4) * t, at1 = ((size_t)u * T + (j1 < T ? j1 : 0)) * D + (D / 4) * t;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t a[4] = {j0 < T ? ld_pair(p.k_tree, at0 + 4 * k, p.f32) : 0u, j1 < T ? ld_pair(p.k_tree, at1 + 4 * k, p.f32) : 0u,
                                           j0 < T ? ld_pair(p.k_tree, at0 + 4 * k + 2, p.f32) : 0u, j1 < T ? ld_pair(p.k_tree, at1 + 4 * k + 2, p.f32) : 0u};
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) mma_bf16(s[mt][nb], a, q[nb][k][0], q[nb][k][1]);
                }
            }
        }
        // visible keys of the chunk for queries 2t and 2t + 1 of the blocks
        if (tree || P - k0 < C::KEYS) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    uint32_t see;
                    if (!tree) {
                        see = (1u << (P - k0)) - 1u;
                    } else {
                        see = 0u;
                        const int r = 8 * nb + 2 * t + e;
                        for (int a = r < R ? r % T : -1; a >= k0;) {   // up the tree, strictly
                            if (a - k0 < 32) see |= 1u << (a - k0);
                            const int up = par[a];
                            a = up < a ? up : -1;
                        }
                    }
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            if (!((see >> (16 * mt + 8 * h + g)) & 1u)) s[mt][nb][2 * h + e] = -INFINITY;
                }
            __syncwarp();
        }
        const float scale = tree ? p.scale_log2 : p.scale_log2 * (1.f / kKv4Unit);
        float mx[NB][2];
        bool grows = false;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float x = fmaxf(fmaxf(s[0][nb][e], s[0][nb][2 + e]), fmaxf(s[1][nb][e], s[1][nb][2 + e]));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
                mx[nb][e] = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16)) * scale;
                grows |= mx[nb][e] > m[nb][e] + (kKv4Shift + 8.f);
            }
        if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float nw = fmaxf(m[nb][e], mx[nb][e] - kKv4Shift);
                    const float a = m[nb][e] == nw ? 1.f : ex2(m[nb][e] - nw);
                    m[nb][e] = nw;
                    l[nb][e] *= a;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) o[i][nb][e] *= a, o[i][nb][2 + e] *= a;
                }
        }
        // P^T's fragments of 16 keys: the accumulators' 8 x 8 tiles transposed
        uint32_t hi[2][NB][2], lo[2][NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            // a query that has seen no key yet: every score is -inf, every probability 0
            const float n0 = m[nb][0] == -INFINITY ? 0.f : -m[nb][0], n1 = m[nb][1] == -INFINITY ? 0.f : -m[nb][1];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float p0 = ex2(fmaf(s[mt][nb][2 * h], scale, n0)), p1 = ex2(fmaf(s[mt][nb][2 * h + 1], scale, n1));
                    l[nb][0] += p0;
                    l[nb][1] += p1;
                    if (tree) p0 *= kKv4Unit, p1 *= kKv4Unit;   // the tree's values are whole: the sums of p v are in units
                    uint32_t a, c2;
                    split_bf16x2_fma(pack2(p0, p1), a, c2);
                    hi[mt][nb][h] = movmatrix(a);
                    lo[mt][nb][h] = movmatrix(c2);
                }
        }
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            auto add_pv = [&](int i, const uint32_t (&a)[4]) {
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    mma_bf16(o[i][nb], a, hi[mt][nb][0], hi[mt][nb][1]);
                    mma_bf16(o[i][nb], a, lo[mt][nb][0], lo[mt][nb][1]);
                }
            };
            if (!tree) {
                Kv4Scale sc[2];
                uint32_t w[4][D / 64];   // rows 2t, 2t + 1 | 2t + 8, 2t + 9 of the 16
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const uint32_t row = 16 * mt + 2 * t + (x & 1) + 8 * (x >> 1);
                    if constexpr (D == 128) {
                        const uint2 v = ld_shared_u64(src + C::CODES + ((row * 64u + g * 8u) ^ (uint32_t)(v_swizzle(row) * 16)));
                        w[x][0] = v.x, w[x][1] = v.y;
                    } else {
                        w[x][0] = ld_shared_u32(src + C::CODES + ((row * 32u + g * 4u) ^ (uint32_t)(v_swizzle(row) * 16)));
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t row = 16 * mt + 2 * t + 8 * h;
                    const uint32_t at = src + C::OFF_SC + 128 + row * 4u;
                    const uint32_t a0 = D == 128 ? at + (g >> 1) : at + (((row ^ odd) & 1u) << 1) + (g >> 2);
                    const uint32_t a1 = D == 128 ? at + 4 + (g >> 1) : at + 4 + ((((row + 1) ^ odd) & 1u) << 1) + (g >> 2);
                    sc[h] = kv4_scales(ld_shared_u8(a0) | ld_shared_u8(a1) << 16);
                }
                // channel i of a word is nibble i / 2 + 4 (i % 2): the low halves of two keys' words
                // side by side hold the even channels, the high halves the odd ones
                if constexpr (D == 128) {
#pragma unroll
                    for (int odd_ch = 0; odd_ch < 2; ++odd_ch) {
                        const uint32_t sel = odd_ch ? 0x7632u : 0x5410u;
                        const uint32_t x0 = __byte_perm(w[0][0], w[1][0], sel), x1 = __byte_perm(w[0][1], w[1][1], sel);
                        const uint32_t x2 = __byte_perm(w[2][0], w[3][0], sel), x3 = __byte_perm(w[2][1], w[3][1], sel);
                        uint32_t v0[4], v1[4], v2[4], v3[4];
                        kv4_word(x0, sc[0], v0), kv4_word(x1, sc[0], v1), kv4_word(x2, sc[1], v2), kv4_word(x3, sc[1], v3);
#pragma unroll
                        for (int n = 0; n < 4; ++n) {
                            const uint32_t a[4] = {v0[n], v1[n], v2[n], v3[n]};
                            add_pv(2 * n + odd_ch, a);
                        }
                    }
                } else {
                    // eight channels a thread: 0..3 in the upper rows, 4..7 in the lower ones
                    const uint32_t e0 = __byte_perm(w[0][0], w[1][0], 0x5410), d0 = __byte_perm(w[0][0], w[1][0], 0x7632);
                    const uint32_t e1 = __byte_perm(w[2][0], w[3][0], 0x5410), d1 = __byte_perm(w[2][0], w[3][0], 0x7632);
                    uint32_t v0[2][4], v1[2][4];
                    kv4_word(e0, sc[0], v0[0]), kv4_word(d0, sc[0], v0[1]), kv4_word(e1, sc[1], v1[0]), kv4_word(d1, sc[1], v1[1]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t a[4] = {v0[i & 1][i >> 1], v0[i & 1][2 + (i >> 1)], v1[i & 1][i >> 1], v1[i & 1][2 + (i >> 1)]};
                        add_pv(i, a);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < D / 16; i += 2) {
                    uint32_t v[2][4];   // channels i, i + 1 (and D / 16 on) of the four keys
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int j = k0 + 16 * mt + 2 * t + (x & 1) + 8 * (x >> 1);
                            v[h][x] = j < T ? ld_pair(p.v_tree, ((size_t)u * T + j) * D + (D / 8) * g + (D / 16) * h + i, p.f32) : 0u;
                        }
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const uint32_t sel = x ? 0x7632u : 0x5410u;
                        const uint32_t a[4] = {__byte_perm(v[0][0], v[0][1], sel), __byte_perm(v[1][0], v[1][1], sel),
                                               __byte_perm(v[0][2], v[0][3], sel), __byte_perm(v[1][2], v[1][3], sel)};
                        add_pv(i + x, a);
                    }
                }
            }
        }
        __syncwarp();   // the stage is read: the next fetch may overwrite it
        stage = stage == C::STAGES - 1 ? 0 : stage + 1;
    }
    cp_async_wait<0>();
    __syncthreads();   // every warp is done with its ring: the states go over it

    constexpr int ROWS = 8 * NB;
    float *st = reinterpret_cast<float *>(smem) + (size_t)warp * ROWS * D;
    float2 *ml = reinterpret_cast<float2 *>(smem + C::OFF_ML);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float x = l[nb][e];
            x += __shfl_xor_sync(0xffffffffu, x, 4);
            x += __shfl_xor_sync(0xffffffffu, x, 8);
            x += __shfl_xor_sync(0xffffffffu, x, 16);
            const int r = 8 * nb + 2 * t + e;
            if (g == 0) ml[warp * ROWS + r] = make_float2(m[nb][e], x);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < D / 16; i += 4)
                    *reinterpret_cast<float4 *>(st + r * D + g * (D / 8) + h * (D / 16) + i) =
                        make_float4(o[i][nb][2 * h + e], o[i + 1][nb][2 * h + e], o[i + 2][nb][2 * h + e], o[i + 3][nb][2 * h + e]);
        }
    __syncthreads();
    // a thread merges four channels of a row at a time
    const bool whole = p.splits == 1;
    for (int i = threadIdx.x; i < R * (D / 4); i += C::THREADS) {
        const int row = i / (D / 4), d = i % (D / 4) * 4;
        float M = -INFINITY, L = 0.f;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int x = 0; x < C::WARPS; ++x) M = fmaxf(M, ml[x * ROWS + row].x);
#pragma unroll
        for (int x = 0; x < C::WARPS; ++x) {
            const float2 y = ml[x * ROWS + row];
            const float w = y.x == -INFINITY ? 0.f : ex2(y.x - M);
            const float4 v = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(smem) + (x * ROWS + row) * D + d);
            L += y.y * w;
            a.x += w * v.x, a.y += w * v.y, a.z += w * v.z, a.w += w * v.w;
        }
        const size_t r = q_row0 + row, part = ((size_t)u * p.splits + split) * R + row;
        if (whole) {
            const float inv = (1.f / kKv4Unit) / L;
            if (d == 0 && p.lse) p.lse[r] = (M + lg2(L)) * 0.69314718055994530942f;
            *reinterpret_cast<uint2 *>(p.out + r * D + d) = make_uint2(bf16x2(a.x * inv, a.y * inv), bf16x2(a.z * inv, a.w * inv));
        } else {
            if (d == 0) p.part_ml[part] = make_float2(M, L);
            *reinterpret_cast<float4 *>(p.part_o + part * D + d) = a;
        }
    }
}

// The parts of split slices: a thread merges four channels of a row, the loads of eight parts
// in flight.
__global__ void __launch_bounds__(128) kv4_merge_kernel(const Kv4AttnParams p, int D)
{
    pdl_release();
    pdl_wait();
    const int per_row = D / 4, rows = (int)blockDim.x / per_row;
    const long long R = (long long)p.G * p.T;
    const long long r = (long long)blockIdx.x * rows + (int)threadIdx.x / per_row;   // row of every slice
    if (r >= p.slices * R) return;
    const int d = ((int)threadIdx.x % per_row) * 4;
    const long long u = r / R, first = u * p.splits * R + (r - u * R);
    float M = -INFINITY, L = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < p.splits; s0 += 8) {
        float2 x[8];
        float4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const long long at = first + min(s0 + i, p.splits - 1) * R;
            x[i] = __ldcg(p.part_ml + at);
            v[i] = __ldcg(reinterpret_cast<const float4 *>(p.part_o + at * D + d));
        }
        float nw = M;
#pragma unroll
        for (int i = 0; i < 8; ++i) nw = fmaxf(nw, x[i].x);
        const float so = M == nw ? 1.f : ex2(M - nw);   // (no part with a key yet: both -inf)
        M = nw;
        L *= so, a.x *= so, a.y *= so, a.z *= so, a.w *= so;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float w = s0 + i >= p.splits || x[i].x == -INFINITY ? 0.f : ex2(x[i].x - M);
            L = fmaf(w, x[i].y, L);
            a.x = fmaf(w, v[i].x, a.x), a.y = fmaf(w, v[i].y, a.y), a.z = fmaf(w, v[i].z, a.z), a.w = fmaf(w, v[i].w, a.w);
        }
    }
    const float inv = (1.f / kKv4Unit) / L;
    if (d == 0 && p.lse) p.lse[r] = (M + lg2(L)) * 0.69314718055994530942f;
    *reinterpret_cast<uint2 *>(p.out + r * D + d) = make_uint2(bf16x2(a.x * inv, a.y * inv), bf16x2(a.z * inv, a.w * inv));
}

template <int D, int NB>
static cudaError_t launch_few_t(const Kv4AttnParams &p, cudaStream_t stream)
{
    using C = Kv4Few<D>;
    static std::atomic<uint64_t> configured{0};
    const cudaError_t e = allow_smem(kv4_attention_few_kernel<D, NB>, C::SMEM, configured);
    if (e != cudaSuccess) return e;
    return launch_chained_smem(kv4_attention_few_kernel<D, NB>, dim3((unsigned)(p.slices * p.splits)), dim3(C::THREADS), dim3(1), C::SMEM,
                               stream, p);
}

cudaError_t launch_kv4_attention(const Kv4AttnParams &p, int D, cudaStream_t stream)
{
    const cudaError_t e = D == 128         ? launch_few_t<128, 1>(p, stream)
                          : p.G * p.T <= 8 ? launch_few_t<64, 1>(p, stream)
                                           : launch_few_t<64, 2>(p, stream);
    if (e != cudaSuccess || p.splits == 1) return e;
    const int rows = 128 / (D / 4);
    const long long n = p.slices * p.G * p.T;
    return launch_chained(kv4_merge_kernel, dim3((unsigned)((n + rows - 1) / rows)), dim3(128), dim3(1), stream, p, D);
}

}  // namespace ppd
