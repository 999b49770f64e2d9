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
        const uint32_t s2 = kv4_scale2(sb[k] * 0x10001u), o2 = kv4_offset2(s2);
        uint32_t v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = kv4_pair(c[k] >> (4 * e), s2, o2);
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

// Blocks of 16 query rows (the G query heads of a K/V head times the T tree tokens) against
// a range of one slice's keys, in registers: four warps take chunks of 32 keys in turn,
//
//   S = Q K^T    mma.sync, K's fragments made from the codes a thread loads: thread t of a
//                quad holds channels [t D / 4, (t + 1) D / 4) of its key, the order of the
//                channels in the sum being free as long as Q follows it
//   O += P V     P from S's accumulators, V's fragments from the codes of two keys at once:
//                columns 2t and 2t + 1 of a block of eight keys are its rows t and t + 4, so
//                that a warp's loads of V meet every bank once
//
// with a running maximum that moves when a score passes it by 2^8, and P as bf16 hi + lo
// (2^-18: V's values are exact, so the output's own rounding is all that shows).  Up to
// eight query rows leave the lower half of a product's 16 rows free: lo goes there and costs
// nothing; more rows take two products.  Each warp's state is merged in shared memory, those of
// a split slice by kv4_merge_kernel.  A chunk's codes and
// scales come by asynchronous copies into a ring of the warp's own: no barrier in the loop.
template <int D>
struct Kv4Few {
    static constexpr int WARPS = 4, THREADS = 128, STAGES = 4, KEYS = 32;
    static constexpr int RB = D / 2;                         // bytes of a row's codes
    static constexpr int SB = D / kKv4Group;                 // scale bytes of a row
    static constexpr uint32_t CODES = KEYS * RB;             // of K, or V, in a stage
    static constexpr uint32_t STAGE = 2 * CODES + 2 * KEYS * 4;
    static constexpr uint32_t OFF_STATE = 0;                 // merge: [WARPS][16][D] over the ring
    static constexpr uint32_t RING = WARPS * STAGES * STAGE;
    static constexpr uint32_t OFF_ML = RING;                 // [WARPS][16]: maximum, sum
    static constexpr uint32_t OFF_PARENT = OFF_ML + WARPS * 16 * 8;
    static constexpr uint32_t SMEM = OFF_PARENT + kMaxTree * 4;
    static_assert(WARPS * 16 * D * 4 <= RING, "the states fit over the ring");
};

template <int D, bool HALF>   // HALF: at most eight rows
__global__ void __launch_bounds__(Kv4Few<D>::THREADS, 3) kv4_attention_few_kernel(const Kv4AttnParams p)
{
    using C = Kv4Few<D>;
    constexpr int NH = HALF ? 1 : 2;   // rows of a thread: g, and g + 8
    extern __shared__ __align__(16) uint8_t smem[];
    pdl_release();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    // row block fastest, then the split, then the slice
    const int rb = (int)(blockIdx.x % p.row_blocks);
    const int us = (int)(blockIdx.x / p.row_blocks), split = us % p.splits;
    const long long u = us / p.splits;
    const int b = (int)(u / p.H % p.B);
    const int T = p.T, R = p.G * T, r0 = rb * 16;
    const int32_t *parent = p.parent + (size_t)b * T;
    const int P_in = ld_input(p.prefix_len + b);
    const int P = min(max(P_in, 0), p.S_max);
    if (u % p.H == 0 && u / p.H < p.B && split == 0 && rb == 0 && warp == 0) {
        const int st = tree_status(parent, T, P_in, p.S_max, lane);
        if (lane == 0) p.dev_status[b] = st;
    }
    int *par = reinterpret_cast<int *>(smem + C::OFF_PARENT);
    for (int i = threadIdx.x; i < T; i += C::THREADS) par[i] = ld_input(parent + i);

    const int n_pref = (P + C::KEYS - 1) / C::KEYS, n_all = n_pref + (T + C::KEYS - 1) / C::KEYS;
    const int c0 = (int)((long long)n_all * split / p.splits), c1 = (int)((long long)n_all * (split + 1) / p.splits);

    const uint32_t ring = smem_addr(smem) + warp * C::STAGES * C::STAGE;
    const size_t row0 = (size_t)u * p.S_max;
    // a chunk's copies: rows past the prefix arrive as zeros (finite: scale 2^-20)
    auto fetch = [&](int c, int stage) {
        if (c < min(c1, n_pref)) {
            const int k0 = c * C::KEYS;
            const uint32_t dst = ring + stage * C::STAGE;
            constexpr int UPR = C::RB / 16;   // 16-byte units of a row
#pragma unroll
            for (int i = 0; i < C::KEYS * UPR / 32; ++i) {
                const int unit = i * 32 + lane, row = unit / UPR;
                const bool in = k0 + row < P;
                const size_t src = (row0 + (in ? k0 : 0)) * C::RB + (in ? unit * 16 : 0);
                const uint32_t uk = unit ^ (((row >> 2) & 1) << 2);
                const uint32_t uv = D == 128 ? unit ^ (((row >> 1) & 1) << 1) : unit;
                cp_async16(dst + uk * 16, p.k_cache + src, in ? 16u : 0u);
                cp_async16(dst + C::CODES + uv * 16, p.v_cache + src, in ? 16u : 0u);
            }
            // a word holds the row's scales (D = 64: those of an even and an odd row; the
            // tensors' last word may be half one)
            const bool in = k0 + lane < P;
            const size_t at = ((row0 + (in ? k0 + lane : 0)) * C::SB) & ~(size_t)3;
            const size_t left = p.scale_bytes - at;
            const uint32_t n = in ? (left < 4 ? (uint32_t)left : 4u) : 0u;
            cp_async4(dst + 2 * C::CODES + lane * 4, p.k_scale + at, n);
            cp_async4(dst + 2 * C::CODES + 128 + lane * 4, p.v_scale + at, n);
        }
        cp_async_commit();
    };
    int next = c0 + warp;   // the next chunk to fetch
#pragma unroll
    for (int s = 0; s < C::STAGES - 1; ++s, next += C::WARPS) fetch(next, s);

    // Q fragments: rows g and g + 8 of the block
    const size_t q_row0 = (size_t)u * R;
    uint32_t q[D / 16][4];
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = h < NH ? r0 + g + 8 * h : R;
            const size_t at = (q_row0 + (r < R ? r : 0)) * D + (D / 4) * t + 4 * s;
            q[s][h] = r < R ? ld_pair(p.q, at, p.f32) : 0u;
            q[s][2 + h] = r < R ? ld_pair(p.q, at + 2, p.f32) : 0u;
        }
    }
    float o[D / 8][4] = {};   // rows g, g + 8; HALF: row g's hi and lo parts
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    __syncthreads();   // the parents are in shared memory

    const int perm = (g >> 1) + 4 * (g & 1);   // key of column g in a block of eight
    int stage = 0;
    for (int c = c0 + warp; c < c1; c += C::WARPS) {
        fetch(next, (stage + C::STAGES - 1) % C::STAGES);
        next += C::WARPS;
        cp_async_wait<C::STAGES - 1>();
        __syncwarp();
        const bool tree = c >= n_pref;
        const int k0 = (tree ? c - n_pref : c) * C::KEYS;
        const uint32_t src = ring + stage * C::STAGE;
        float s[4][4] = {};
        if (!tree) {
            const uint32_t ks = ld_shared_u32(src + 2 * C::CODES + lane * 4) >>
                                (D == 64 ? (uint32_t)((row0 + k0 + lane) & 1) * 16u : 0u);
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int row = 8 * n + perm;
                const uint32_t sw = __shfl_sync(0xffffffffu, ks, row);
                const uint32_t s2 = kv4_scale2(((sw >> (D == 128 ? 8 * t : 8 * (t >> 1))) & 0xFFu) * 0x10001u);
                const uint32_t o2 = kv4_offset2(s2);
                uint32_t w[D / 32];
                const uint32_t x = ((row >> 2) & 1) * 64u;
                if constexpr (D == 128) {
                    const uint4 v = ld_shared_u128(src + (((uint32_t)row * 64u + t * 16u) ^ x));
                    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
                } else {
                    const uint2 v = ld_shared_u64(src + (((uint32_t)row * 32u + t * 8u) ^ x));
                    w[0] = v.x, w[1] = v.y;
                }
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    mma_bf16(s[n], q[k], kv4_pair(w[k >> 1] >> (8 * (k & 1)), s2, o2),
                             kv4_pair(w[k >> 1] >> (8 * (k & 1) + 4), s2, o2));
            }
        } else {
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int j = k0 + 8 * n + perm;
                const size_t at = ((size_t)u * T + (j < T ? j : 0)) * D + (D / 4) * t;
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    mma_bf16(s[n], q[k], j < T ? ld_pair(p.k_tree, at + 4 * k, p.f32) : 0u,
                             j < T ? ld_pair(p.k_tree, at + 4 * k + 2, p.f32) : 0u);
            }
        }
        // visible keys of the chunk for rows g and g + 8
        uint32_t see[2];
        if (!tree) {
            see[0] = see[1] = P - k0 >= 32 ? 0xffffffffu : (1u << (P - k0)) - 1u;
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = h < NH ? r0 + g + 8 * h : R;
                see[h] = 0u;
                for (int a = r < R ? r % T : -1; a >= k0;) {   // up the tree, strictly
                    if (a - k0 < 32) see[h] |= 1u << (a - k0);
                    const int up = par[a];
                    a = up < a ? up : -1;
                }
            }
        }
        if (__any_sync(0xffffffffu, (see[0] & see[1]) != 0xffffffffu)) {
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int e = 0; e < 2 * NH; ++e)
                    if (!((see[e >> 1] >> (8 * n + t + 4 * (e & 1))) & 1u)) s[n][e] = -INFINITY;
        }
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int h = 0; h < NH; ++h) {
#pragma unroll
            for (int n = 0; n < 4; ++n) mx[h] = max3(mx[h], s[n][2 * h], s[n][2 * h + 1]);
            mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
            mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2)) * p.scale_log2;
        }
        if (__any_sync(0xffffffffu, mx[0] > m[0] + 8.f || mx[1] > m[1] + 8.f)) {
            float a[2];
#pragma unroll
            for (int h = 0; h < NH; ++h) {
                const float nw = fmaxf(m[h], mx[h]);
                a[h] = m[h] == nw ? 1.f : ex2(m[h] - nw);
                m[h] = nw;
                l[h] *= a[h];
            }
            if (HALF) a[1] = a[0];
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][e] *= a[e >> 1];
        }
        // a row that has seen no key yet: every score is -inf, every probability 0
        const float nm[2] = {m[0] == -INFINITY ? 0.f : -m[0], m[1] == -INFINITY ? 0.f : -m[1]};
        // P's fragments of 16 keys: hi and lo in the two halves of the rows, or one after the other
        uint32_t pa[2][HALF ? 1 : 2][4];
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int h = 0; h < NH; ++h) {
                const float p0 = ex2(fmaf(s[n][2 * h], p.scale_log2, nm[h])), p1 = ex2(fmaf(s[n][2 * h + 1], p.scale_log2, nm[h]));
                l[h] += p0 + p1;
                uint32_t hi, lo;
                split_bf16x2(pack2(p0, p1), p0, p1, hi, lo);
                pa[n >> 1][0][2 * (n & 1) + h] = hi;
                if (HALF) pa[n >> 1][0][2 * (n & 1) + 1] = lo;
                else pa[n >> 1][NH - 1][2 * (n & 1) + h] = lo;
            }
        auto add_pv = [&](int kk, float (&acc)[4], uint32_t b0, uint32_t b1) {
            mma_bf16(acc, pa[kk][0], b0, b1);
            if (!HALF) mma_bf16(acc, pa[kk][NH - 1], b0, b1);
        };
        // O += P V, 16 keys at a time: rows t, t + 4 | t + 8, t + 12 of the 16
        if (!tree) {
            const uint32_t vs = ld_shared_u32(src + 2 * C::CODES + 128 + lane * 4) >>
                                (D == 64 ? (uint32_t)((row0 + k0 + lane) & 1) * 16u : 0u);
            const uint32_t v0 = src + C::CODES;
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                uint32_t w[4][D / 64], s2[2], o2[2];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t row = 16 * kk + t + 4 * i;
                    if constexpr (D == 128) {
                        const uint2 v = ld_shared_u64(v0 + ((row * 64u + g * 8u) ^ (((row >> 1) & 1) * 32u)));
                        w[i][0] = v.x, w[i][1] = v.y;
                    } else {
                        w[i][0] = ld_shared_u32(v0 + row * 32u + g * 4u);
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t sa = __shfl_sync(0xffffffffu, vs, 16 * kk + t + 8 * i);
                    const uint32_t sb = __shfl_sync(0xffffffffu, vs, 16 * kk + t + 8 * i + 4);
                    const uint32_t sh = D == 128 ? 8 * (g >> 1) : 8 * (g >> 2);
                    s2[i] = kv4_scale2(((sa >> sh) & 0xFFu) | ((sb >> sh) & 0xFFu) << 16);
                    o2[i] = kv4_offset2(s2[i]);
                }
#pragma unroll
                for (int x = 0; x < D / 64; ++x) {
#pragma unroll
                    for (int half = 0; half < 2; ++half) {   // nibbles 0..3, then 4..7
                        const uint32_t sel = half ? 0x7632u : 0x5410u;
                        const uint32_t c0w = __byte_perm(w[0][x], w[1][x], sel), c1w = __byte_perm(w[2][x], w[3][x], sel);
#pragma unroll
                        for (int n = 0; n < 4; ++n)   // nibble n + 4 half: channel 2 n + half of the word
                            add_pv(kk, o[8 * x + 2 * n + half], kv4_pair(c0w >> (4 * n), s2[0], o2[0]),
                                   kv4_pair(c1w >> (4 * n), s2[1], o2[1]));
                    }
                }
            }
        } else {
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int i = 0; i < D / 8; i += 2) {   // channels i, i + 1 of g's
                    uint32_t v[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int j = k0 + 16 * kk + t + 4 * x;
                        v[x] = j < T ? ld_pair(p.v_tree, ((size_t)u * T + j) * D + (D / 8) * g + i, p.f32) : 0u;
                    }
                    add_pv(kk, o[i], __byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410));
                    add_pv(kk, o[i + 1], __byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632));
                }
        }
        __syncwarp();   // the stage is read: the next fetch may overwrite it
        stage = (stage + 1) % C::STAGES;
    }
    cp_async_wait<0>();
    __syncthreads();   // every warp is done with its ring: the states go over it

    float *st = reinterpret_cast<float *>(smem) + (size_t)warp * 16 * D;
    float2 *ml = reinterpret_cast<float2 *>(smem + C::OFF_ML);
    if (HALF) {
#pragma unroll
        for (int i = 0; i < D / 8; ++i) o[i][0] += o[i][2], o[i][1] += o[i][3];
    }
#pragma unroll
    for (int h = 0; h < NH; ++h) {
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
        if (t == 0) ml[warp * 16 + g + 8 * h] = make_float2(m[h], l[h]);
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < D / 8; i += 4)
                *reinterpret_cast<float4 *>(st + (g + 8 * h) * D + (2 * t + e) * (D / 8) + i) =
                    make_float4(o[i][2 * h + e], o[i + 1][2 * h + e], o[i + 2][2 * h + e], o[i + 3][2 * h + e]);
    }
    __syncthreads();
    // a thread merges D / 8 channels of a row
    const int row = threadIdx.x >> 3, d0 = (threadIdx.x & 7) * (D / 8);
    if (row >= 8 * NH || r0 + row >= R) return;
    float M = -INFINITY, w[C::WARPS], L = 0.f;
#pragma unroll
    for (int i = 0; i < C::WARPS; ++i) M = fmaxf(M, ml[i * 16 + row].x);
#pragma unroll
    for (int i = 0; i < C::WARPS; ++i) {
        const float2 x = ml[i * 16 + row];
        w[i] = x.x == -INFINITY ? 0.f : ex2(x.x - M);
        L += x.y * w[i];
    }
    const size_t r = q_row0 + r0 + row;
    const bool whole = p.splits == 1;
    const float inv = whole ? 1.f / L : 1.f;
    const long long part = (u * p.splits + split) * R + r0 + row;
    if (d0 == 0) {
        if (whole) {
            if (p.lse) p.lse[r] = (M + lg2(L)) * 0.69314718055994530942f;
        } else {
            p.part_ml[part] = make_float2(M, L);
        }
    }
#pragma unroll
    for (int i = 0; i < D / 8; i += 4) {
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int x = 0; x < C::WARPS; ++x) {
            const float4 v = *reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(smem) + (size_t)x * 16 * D + row * D + d0 + i);
            a.x += w[x] * v.x, a.y += w[x] * v.y, a.z += w[x] * v.z, a.w += w[x] * v.w;
        }
        if (whole) {
            const uint2 v = make_uint2(bf16x2(a.x * inv, a.y * inv), bf16x2(a.z * inv, a.w * inv));
            *reinterpret_cast<uint2 *>(p.out + r * D + d0 + i) = v;
        } else {
            *reinterpret_cast<float4 *>(p.part_o + part * D + d0 + i) = a;
        }
    }
}

// The parts of split slices: a thread merges four channels of a row.
__global__ void __launch_bounds__(256) kv4_merge_kernel(const Kv4AttnParams p, int D)
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
    for (int s = 0; s < p.splits; ++s) M = fmaxf(M, p.part_ml[first + s * R].x);
    for (int s = 0; s < p.splits; ++s) {
        const float2 x = p.part_ml[first + s * R];
        if (x.x == -INFINITY) continue;
        const float w = ex2(x.x - M);
        const float4 v = *reinterpret_cast<const float4 *>(p.part_o + (first + s * R) * D + d);
        L += x.y * w;
        a.x += w * v.x, a.y += w * v.y, a.z += w * v.z, a.w += w * v.w;
    }
    const float inv = 1.f / L;
    if (d == 0 && p.lse) p.lse[r] = (M + lg2(L)) * 0.69314718055994530942f;
    *reinterpret_cast<uint2 *>(p.out + r * D + d) = make_uint2(bf16x2(a.x * inv, a.y * inv), bf16x2(a.z * inv, a.w * inv));
}

template <int D, bool HALF>
static cudaError_t launch_few_t(const Kv4AttnParams &p, cudaStream_t stream)
{
    using C = Kv4Few<D>;
    static std::atomic<uint64_t> configured{0};
    const cudaError_t e = allow_smem(kv4_attention_few_kernel<D, HALF>, C::SMEM, configured);
    if (e != cudaSuccess) return e;
    return launch_chained_smem(kv4_attention_few_kernel<D, HALF>, dim3((unsigned)(p.slices * p.splits * p.row_blocks)),
                               dim3(C::THREADS), dim3(1), C::SMEM, stream, p);
}

cudaError_t launch_kv4_attention(const Kv4AttnParams &p, int D, cudaStream_t stream)
{
    const bool half = p.G * p.T <= 8;
    const cudaError_t e = D == 128 ? (half ? launch_few_t<128, true>(p, stream) : launch_few_t<128, false>(p, stream))
                                   : (half ? launch_few_t<64, true>(p, stream) : launch_few_t<64, false>(p, stream));
    if (e != cudaSuccess || p.splits == 1) return e;
    const int rows = 256 / (D / 4);
    const long long n = p.slices * p.G * p.T;
    return launch_chained(kv4_merge_kernel, dim3((unsigned)((n + rows - 1) / rows)), dim3(256), dim3(1), stream, p, D);
}

}  // namespace ppd
