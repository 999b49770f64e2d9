// ppd_evict.cu -- a cache cut down by attention weight: the weight that accepted tokens
// gave each cached row, added up (ppd_kv_weight_add), and the rows kept (ppd_kv_evict).
#include "ppd_kv4.cuh"

namespace ppd {

// ------------------------------------------------------------------ weight per cached row

// A warp takes chunks of 32 keys of a slice: S^T = K Q^T by mma.sync for the slice's G n accepted
// query rows in blocks of eight (their fragments in shared memory, up to 32 rows at a time),
// p = exp(scale S - lse), and each key's sum over the rows: the columns of a thread, then a
// halving exchange over a quad that leaves one key to each lane.  K's fragments are made from the
// codes (or bf16 channels) that asynchronous copies bring into a ring of the warp's own; the
// order of the channels in the sum is free as long as Q follows it.  Tree keys come last: the
// path's own rows, each seen by itself and the nodes after it.
//
// A bf16 cache: bound by HBM, 1.38 GB (B = 8, up to 16,384 keys, 16 heads of two) 208 us, 6.6 TB/s.
// 4 bits: by a warp's chain from codes to products (issue slots 50 % used, the tensor pipe 15 %) and by
// the second wave of blocks, two thirds full: 1024 slices of 2048 keys 51 us, 3.2 TB/s (the bf16 cache 95 us).
constexpr int kWeightRows = 32;

template <int D, bool KV4>
struct KvWeight {
    static constexpr int BLOCKS = KV4 ? 4 : 3;                         // on an SM
    static constexpr int STAGES = KV4 ? 4 : (D == 128 ? 2 : 4);
    static constexpr uint32_t RB = KV4 ? D / 2 : 2 * D;                // bytes of a row
    static constexpr uint32_t STAGE = 32 * RB + (KV4 ? 128 : 0);       // rows, then a word of scales each
    static constexpr uint32_t OFF_Q = 4 * STAGES * STAGE;
    static constexpr uint32_t SMEM = OFF_Q + kWeightRows / 8 * (D / 16) * 32 * 8;
};

template <int D, bool KV4>
__global__ void __launch_bounds__(128, (KvWeight<D, KV4>::BLOCKS)) kv_weight_kernel(const KvWeightParams p)
{
    using C = KvWeight<D, KV4>;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int path_s[kMaxTree];
    __shared__ __align__(16) float neg_lse[kWeightRows];
    __shared__ __align__(8) int place[kWeightRows];   // of the rows on the path; -1: none, no row of its own
    uint2 (*q_s)[D / 16][32] = reinterpret_cast<uint2(*)[D / 16][32]>(smem + C::OFF_Q);
    pdl_release();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int split = (int)(blockIdx.x % p.splits);
    const uint32_t u = blockIdx.x / p.splits;
    const int b = (int)(u / (uint32_t)p.H % (uint32_t)p.B);
    const int T = p.T;
    const int P = ld_input(p.prefix_len + b);
    const int n = min(ld_input(p.accept_len + b), T);
    if (n < 1 || P < 0 || P > p.S_max) return;   // uniform over the block
    const int n_pref = (P + 31) / 32, n_all = n_pref + (n + 31) / 32;
    const int c0 = (int)((long long)n_all * split / p.splits), c1 = (int)((long long)n_all * (split + 1) / p.splits);
    const int rows = p.G * n;
    const size_t row0 = (size_t)u * p.S_max;
    // first channel of step s of a quad's thread: as the thread's loads of K bring them
    auto channel = [&](int s) { return KV4 ? (D / 4) * t + 4 * s : 32 * (s >> 1) + 8 * t + 4 * (s & 1); };

    const uint32_t ring = smem_addr(smem) + warp * C::STAGES * C::STAGE;
    constexpr int UPR = C::RB / 16;   // 16-byte pieces of a row; bf16: the odd rows' halves of 128 bytes change places
    // piece i of a lane is 512 bytes (an even number of rows) on from piece i - 1
    const uint32_t to = (uint32_t)(lane ^ (KV4 ? 0 : (lane / UPR & 1) << 2)) * 16;
    auto fetch = [&](int c, int stage) {
        if (c < min(c1, n_pref)) {
            const int k0 = c * 32, left_rows = P - k0;
            const uint32_t dst = ring + stage * C::STAGE;
            const uint8_t *src = p.k_cache + (row0 + k0) * C::RB + lane * 16;
            constexpr int SB = D / kKv4Group;
            if (left_rows >= 32 && !(KV4 && D == 64)) {
#pragma unroll
                for (int i = 0; i < UPR; ++i) cp_async16(dst + to + i * 512, src + i * 512, 16u);
                if (KV4) cp_async4(dst + 32 * C::RB + lane * 4, p.k_scale + (row0 + k0 + lane) * SB, 4u);
            } else {
#pragma unroll
                for (int i = 0; i < UPR; ++i) {
                    const int row = (i * 32 + lane) / UPR;
                    const bool in = row < left_rows;   // rows past the prefix arrive as zeros
                    cp_async16(dst + to + i * 512, in ? src + i * 512 : p.k_cache, in ? 16u : 0u);
                }
                if constexpr (KV4) {   // (D = 64: a word holds an even and an odd row's scales, the tensor's last perhaps one)
                    const bool in = lane < left_rows;
                    const size_t a = ((row0 + (in ? k0 + lane : 0)) * SB) & ~(size_t)3;
                    const size_t left = p.scale_bytes - a;
                    cp_async4(dst + 32 * C::RB + lane * 4, p.k_scale + a, in ? (left < 4 ? (uint32_t)left : 4u) : 0u);
                }
            }
        }
        cp_async_commit();
    };
    for (int i = threadIdx.x; i < n; i += 128) path_s[i] = ld_input(p.path + (size_t)b * T + i);

    for (int r0 = 0; r0 < rows; r0 += kWeightRows) {
        __syncthreads();   // the path is there; the rows before these are done with
        int next = c0 + warp;   // the next chunk to fetch
#pragma unroll
        for (int s = 0; s < C::STAGES - 1; ++s, next += 4) fetch(next, s);
        const int blocks = (min(kWeightRows, rows - r0) + 7) / 8;
        for (int x = warp; x < blocks; x += 4) {
            const int r = r0 + 8 * x + g, a = r % n, node = r < rows ? path_s[a] : -1;
            const bool real = node >= 0 && node < T;
            const size_t row = ((size_t)u * p.G + (real ? r / n : 0)) * T + (real ? node : 0);
#pragma unroll
            for (int s = 0; s < D / 16; ++s)
                q_s[x][s][lane] = real ? make_uint2(ld_pair(p.q, row * D + channel(s), p.f32), ld_pair(p.q, row * D + channel(s) + 2, p.f32))
                                       : make_uint2(0u, 0u);
            if (t == 0) {
                neg_lse[8 * x + g] = real ? -1.4426950408889634f * ld_input(p.lse + row) : -INFINITY;
                place[8 * x + g] = real ? a : -1;
            }
        }
        __syncthreads();
        int stage = 0;
        for (int c = c0 + warp; c < c1; c += 4) {
            fetch(next, stage == 0 ? C::STAGES - 1 : stage - 1);
            next += 4;
            const bool tree = c >= n_pref;
            const int k0 = (tree ? c - n_pref : c) * 32;
            const int mine = k0 + 8 * t + g;   // this lane's key in the end
            const bool stays = tree ? mine < n && P + mine < p.S_max : mine < P;
            float *out = p.weight + row0 + (tree ? P : 0) + (stays ? mine : 0);
            float old = 0.f;
            if (stays && (!tree || r0 > 0)) old = ld_input(out);
            uint32_t k[2][D / 16][4];   // K's fragments of 2 x 16 keys
            if (tree) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int a = k0 + 8 * i + g, node = a < n ? path_s[a] : -1;
                    const bool real = node >= 0 && node < T;
                    const size_t row = ((size_t)u * T + (real ? node : 0)) * D;
#pragma unroll
                    for (int s = 0; s < D / 16; ++s) {
                        k[i >> 1][s][i & 1] = real ? ld_pair(p.k_tree, row + channel(s), p.f32) : 0u;
                        k[i >> 1][s][2 + (i & 1)] = real ? ld_pair(p.k_tree, row + channel(s) + 2, p.f32) : 0u;
                    }
                }
            } else {
                cp_async_wait<C::STAGES - 1>();
                __syncwarp();
                const uint32_t src = ring + stage * C::STAGE;
                const uint32_t odd = D == 64 ? (uint32_t)(row0 + k0) & 1u : 0u;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t row = 8 * i + g;
                    if constexpr (KV4) {
                        uint32_t w[D / 32];
                        if constexpr (D == 128) {
                            const uint4 v = ld_shared_u128(src + row * 64u + t * 16u);
                            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
                        } else {
                            const uint2 v = ld_shared_u64(src + row * 32u + t * 8u);
                            w[0] = v.x, w[1] = v.y;
                        }
                        const uint32_t at = D == 128 ? t : (((row ^ odd) & 1u) << 1) + (t >> 1);
                        const Kv4Scale sc = kv4_scales(ld_shared_u8(src + 32 * C::RB + row * 4u + at) * 0x10001u);
#pragma unroll
                        for (int x = 0; x < D / 32; ++x) {
                            uint32_t v[4];
                            kv4_word(w[x], sc, v);
                            k[i >> 1][2 * x][i & 1] = v[0], k[i >> 1][2 * x][2 + (i & 1)] = v[1];
                            k[i >> 1][2 * x + 1][i & 1] = v[2], k[i >> 1][2 * x + 1][2 + (i & 1)] = v[3];
                        }
                    } else {
#pragma unroll
                        for (int x = 0; x < D / 32; ++x) {
                            const uint4 v = ld_shared_u128(src + row * C::RB + (uint32_t)((4 * x + t) ^ ((row & 1) << 2)) * 16);
                            k[i >> 1][2 * x][i & 1] = v.x, k[i >> 1][2 * x][2 + (i & 1)] = v.y;
                            k[i >> 1][2 * x + 1][i & 1] = v.z, k[i >> 1][2 * x + 1][2 + (i & 1)] = v.w;
                        }
                    }
                }
            }
            const float scale = KV4 && !tree ? p.scale_log2 * (1.f / kKv4Unit) : p.scale_log2;
            float sum[4] = {0.f, 0.f, 0.f, 0.f};   // keys g, g + 8, g + 16, g + 24
#pragma unroll 1
            for (int x = 0; x < blocks; ++x) {
                float s[2][4] = {};
#pragma unroll
                for (int y = 0; y < D / 16; ++y) {
                    const uint2 q = q_s[x][y][lane];
                    mma_bf16(s[0], k[0][y], q.x, q.y);
                    mma_bf16(s[1], k[1][y], q.x, q.y);
                }
                const float2 nl = *reinterpret_cast<const float2 *>(neg_lse + 8 * x + 2 * t);
                if (KV4 && !tree) {   // (a row that is none: products of zeros and finite values)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        sum[i] += ex2(fmaf(s[i >> 1][2 * (i & 1)], scale, nl.x)) + ex2(fmaf(s[i >> 1][2 * (i & 1) + 1], scale, nl.y));
                } else {
                    const int2 at = *reinterpret_cast<const int2 *>(place + 8 * x + 2 * t);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {   // a later node's row is not seen, and a row that is none sees nothing (0 times an infinity)
                        const int key = tree ? k0 + 8 * i + g : 0;
                        if (at.x >= key) sum[i] += ex2(fmaf(s[i >> 1][2 * (i & 1)], scale, nl.x));
                        if (at.y >= key) sum[i] += ex2(fmaf(s[i >> 1][2 * (i & 1) + 1], scale, nl.y));
                    }
                }
            }
            // four values over the four lanes of a quad: lane t ends with value t
#pragma unroll
            for (int half = 2; half >= 1; half >>= 1) {
                const bool up = (t & half) != 0;
#pragma unroll
                for (int i = 0; i < half; ++i) {
                    const float send = up ? sum[i] : sum[i + half], keep = up ? sum[i + half] : sum[i];
                    sum[i] = keep + __shfl_xor_sync(0xffffffffu, send, half);
                }
            }
            if (stays) *out = old + sum[0];
            __syncwarp();   // the stage is read: the next fetch may overwrite it
            stage = stage == C::STAGES - 1 ? 0 : stage + 1;
        }
        cp_async_wait<0>();
    }
}

template <int D, bool KV4>
static cudaError_t launch_weight_t(const KvWeightParams &p, cudaStream_t stream)
{
    using C = KvWeight<D, KV4>;
    static std::atomic<uint64_t> configured{0};
    const cudaError_t e = allow_smem(kv_weight_kernel<D, KV4>, C::SMEM, configured);
    if (e != cudaSuccess) return e;
    return launch_chained_smem(kv_weight_kernel<D, KV4>, dim3((unsigned)(p.slices * p.splits)), dim3(128), dim3(1), C::SMEM, stream, p);
}

int kv_weight_blocks(bool kv4) { return kv4 ? 4 : 3; }

cudaError_t launch_kv_weight(const KvWeightParams &p, int D, cudaStream_t stream)
{
    if (p.k_scale) return D == 128 ? launch_weight_t<128, true>(p, stream) : launch_weight_t<64, true>(p, stream);
    return D == 128 ? launch_weight_t<128, false>(p, stream) : launch_weight_t<64, false>(p, stream);
}

// ------------------------------------------------------------------ the rows to keep

constexpr int kSelThreads = 512, kSelBins = 2048;

// Weights in order as unsigned numbers (-0 as +0); a NaN above every number.
PPD_DEV uint32_t weight_rank(float w)
{
    if (w != w) return 0xFFFFFFFEu;
    const uint32_t x = __float_as_uint(w + 0.f);
    return x & 0x80000000u ? ~x : x | 0x80000000u;
}

// One block per slice: the rank of the last row kept, by counting digits of 11, 11 and 10 bits
// from the top, then the kept rows' indices in order: all above that rank, and of those equal
// to it the first ones.  The first and last rows rank above all.  Ranks are read once and
// stay in shared memory where they fit (CACHED); after the first digit the rows that share
// it are a short list in most cases, which the other digits are counted on.  The indices need
// no barrier in their loop: each warp counts its stretch of the rows, then writes it.
// Bound by the chain of digits and barriers: 1024 slices of up to 16,384 rows, seven waves of
// blocks, are a fifth of an eviction's 285 us.
constexpr int kSelList = 2048, kSelWarps = kSelThreads / 32;

template <bool CACHED>
__global__ void __launch_bounds__(kSelThreads) kv_select_kernel(const KvEvictParams p)
{
    extern __shared__ uint32_t ranks[];
    __shared__ uint32_t hist[kSelBins], list[kSelList];
    __shared__ uint32_t warp_sum[kSelWarps], warp_eq[kSelWarps];
    __shared__ uint32_t found[3], n_list;   // the bin, how many rows rank above it, how many share it
    pdl_release();
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t u = blockIdx.x;
    const int b = (int)(u / (uint32_t)p.H % (uint32_t)p.B);
    const int len = ld_input(p.length + b);
    const bool bad = len < 0 || len > p.S_max;
    if (u / p.H < p.B && u % p.H == 0 && tid == 0) {
        p.dev_status[b] = bad ? kErrCapacity : kOk;
        p.new_len[b] = bad ? len : min(len, p.budget);
    }
    int32_t *kept = p.kept + (size_t)u * p.budget;
    if (bad || len <= p.budget) {
        for (int i = tid; i < p.budget; i += kSelThreads) kept[i] = !bad && i < len ? i : -1;
        return;
    }
    const float *w = p.weight + (size_t)u * p.S_max;
    auto rank_of = [&](int j) {
        return j < p.sink || j >= len - p.recent ? 0xFFFFFFFFu : weight_rank(ld_input(w + j));
    };
    auto rank = [&](int j) { return CACHED ? ranks[j] : rank_of(j); };
    for (int i = tid; i < kSelBins; i += kSelThreads) hist[i] = 0;
    if (tid == 0) n_list = 0;
    __syncthreads();
    auto take = [&](int j, float x) {
        const uint32_t r = j < p.sink || j >= len - p.recent ? 0xFFFFFFFFu : weight_rank(x);
        if (CACHED) ranks[j] = r;
        atomicAdd(hist + (r >> 21), 1u);
    };
    // 32 bytes or more a thread in flight
    const int len4 = (reinterpret_cast<uintptr_t>(w) & 15) == 0 ? len / 4 : 0;
    for (int i0 = tid; i0 < len4; i0 += 4 * kSelThreads) {
        float4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = i0 + i * kSelThreads < len4 ? ld_input(reinterpret_cast<const float4 *>(w) + i0 + i * kSelThreads) : float4{};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = 4 * (i0 + i * kSelThreads);
            if (j < 4 * len4) take(j, x[i].x), take(j + 1, x[i].y), take(j + 2, x[i].z), take(j + 3, x[i].w);
        }
    }
    for (int j0 = 4 * len4 + tid; j0 < len; j0 += 8 * kSelThreads) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = j0 + i * kSelThreads < len ? ld_input(w + j0 + i * kSelThreads) : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (j0 + i * kSelThreads < len) take(j0 + i * kSelThreads, x[i]);
    }
    uint32_t prefix = 0, need = (uint32_t)p.budget;   // of the rows with the digits found so far, `need` are kept
    bool listed = false;
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
        const int bits = round < 2 ? 11 : 10, bins = 1 << bits, shift = round == 0 ? 21 : round == 1 ? 10 : 0;
        if (round > 0) {
            const uint32_t above = 0xFFFFFFFFu << (shift + bits);
            for (int i = tid; i < kSelBins; i += kSelThreads) hist[i] = 0;
            __syncthreads();
            const int n = listed ? (int)n_list : len;
            for (int j = tid; j < n; j += kSelThreads) {
                const uint32_t r = listed ? list[j] : rank(j);
                if ((r & above) == prefix) atomicAdd(hist + ((r >> shift) & (bins - 1)), 1u);
            }
        }
        __syncthreads();
        // rows ranking in a higher bin, from the top: thread i has bins 4 i .. of the order
        constexpr int per = kSelBins / kSelThreads;
        uint32_t c[per], s = 0;
#pragma unroll
        for (int i = 0; i < per; ++i) {
            const int bin = bins - 1 - (tid * per + i);
            c[i] = bin >= 0 ? hist[bin] : 0u;
            s += c[i];
        }
        uint32_t inc = s;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += x;
        }
        if (lane == 31) warp_sum[warp] = inc;
        __syncthreads();
        uint32_t before = inc - s;
        for (int i = 0; i < warp; ++i) before += warp_sum[i];
#pragma unroll
        for (int i = 0; i < per; ++i) {
            if (before < need && need <= before + c[i]) {
                found[0] = (uint32_t)(bins - 1 - (tid * per + i));
                found[1] = before;
                found[2] = c[i];
            }
            before += c[i];
        }
        __syncthreads();
        prefix |= found[0] << shift;
        need -= found[1];
        if (round == 0 && found[2] <= kSelList) {
            listed = true;
            for (int j = tid; j < len; j += kSelThreads) {
                const uint32_t r = rank(j);
                if (r >> 21 == prefix >> 21) list[atomicAdd(&n_list, 1u)] = r;
            }
        }
        __syncthreads();
    }
    // a warp's stretch of rows: how many rank above `prefix`, how many equal it
    const int stretch = ((len + kSelThreads - 1) / kSelThreads) * 32;
    const int j0 = min(len, warp * stretch), j1 = min(len, j0 + stretch);
    uint32_t n_gt = 0, n_eq = 0;
    for (int j = j0 + lane; j < j1; j += 32) {
        const uint32_t r = rank(j);
        n_gt += r > prefix;
        n_eq += r == prefix;
    }
    n_gt = __reduce_add_sync(0xffffffffu, n_gt);
    n_eq = __reduce_add_sync(0xffffffffu, n_eq);
    if (lane == 0) warp_sum[warp] = n_gt, warp_eq[warp] = n_eq;
    __syncthreads();
    uint32_t out = 0, eq = 0;   // kept rows before this warp's, and equal ones before it
    for (int i = 0; i < warp; ++i) out += warp_sum[i], eq += warp_eq[i];
    out += min(eq, need);
    for (int j = j0; j < j1; j += 32) {
        const uint32_t r = j + lane < j1 ? rank(j + lane) : 0u;
        const uint32_t is_gt = __ballot_sync(0xffffffffu, j + lane < j1 && r > prefix);
        uint32_t is_eq = __ballot_sync(0xffffffffu, j + lane < j1 && r == prefix);
        const uint32_t low = (1u << lane) - 1u;
        // of the equal rows the first ones, until there are `need`
        const uint32_t left = need > eq ? need - eq : 0u;
        eq += __popc(is_eq);
        is_eq = __ballot_sync(0xffffffffu, ((is_eq >> lane) & 1u) && __popc(is_eq & low) < left);
        const uint32_t take = is_gt | is_eq;
        if ((take >> lane) & 1u) kept[out + __popc(take & low)] = j + lane;
        out += __popc(take);
    }
}

// ------------------------------------------------------------------ moving them

template <int BYTES>
struct MoveUnit;
template <> struct MoveUnit<16> { using T = uint4; };
template <> struct MoveUnit<8> { using T = uint2; };
template <> struct MoveUnit<4> { using T = uint32_t; };
template <> struct MoveUnit<2> { using T = uint16_t; };
template <> struct MoveUnit<1> { using T = uint8_t; };

constexpr int kMoveThreads = 256, kMoveDeep = 4;

// Kept row i goes to row i of the destination: each step of a block reads kMoveDeep units a thread
// (16 bytes where rows and addresses allow), then writes them; the next step's row indices are on
// their way meanwhile.  In place a block takes its columns of the whole slice alone, in order:
// the rows of a step lie at or above their places, and so do those of every later step, so
// what a step overwrites has been read.  Bound by HBM, which brings 128 bytes for a row of 64 that
// lies alone: 4096 of 16,384 rows kept, 1024 slices of a 4-bit cache, four fifths of the call's 285 us,
// in which 1.5 GB are read and written for 1.2 that are needed.
template <int BYTES, int THREADS>   // 32: a warp, else a block
PPD_DEV void move_rows(const KvEvictParams &p, const KvPlane &pl, const int32_t *kept, uint32_t u, int c0, int c1, int i0, int i1, int tid)
{
    using T = typename MoveUnit<BYTES>::T;
    const int per_row = pl.row_bytes / BYTES, w = c1 - c0;   // this block's units of a row
    const T *src = reinterpret_cast<const T *>(static_cast<const uint8_t *>(pl.src) + (size_t)u * p.S_max * pl.row_bytes) + c0;
    T *dst = reinterpret_cast<T *>(static_cast<uint8_t *>(pl.dst) + (size_t)u * p.S_out * pl.row_bytes) + c0;
    const bool in_place = pl.src == pl.dst;
    const int rows = THREADS * kMoveDeep / w;           // of a step
    int row[kMoveDeep], col[kMoveDeep], from[kMoveDeep];
#pragma unroll
    for (int x = 0; x < kMoveDeep; ++x) {
        const int unit = x * THREADS + tid;
        row[x] = unit / w;
        col[x] = unit - row[x] * w;
        if (row[x] >= rows) row[x] = i1;   // none
        from[x] = i0 + row[x] < i1 ? kept[i0 + row[x]] : -1;
    }
    for (int r0 = i0; r0 < i1; r0 += rows) {
        T v[kMoveDeep];
        bool go[kMoveDeep];
#pragma unroll
        for (int x = 0; x < kMoveDeep; ++x) {
            go[x] = from[x] >= 0 && !(in_place && from[x] == r0 + row[x]);
            if (go[x]) v[x] = src[(size_t)from[x] * per_row + col[x]];
        }
#pragma unroll
        for (int x = 0; x < kMoveDeep; ++x) from[x] = r0 + rows + row[x] < i1 ? kept[r0 + rows + row[x]] : -1;
        if (in_place) {
            if (THREADS == 32) __syncwarp();
            else __syncthreads();
        }
#pragma unroll
        for (int x = 0; x < kMoveDeep; ++x)
            if (go[x]) dst[(size_t)(r0 + row[x]) * per_row + col[x]] = v[x];
    }
}

template <int THREADS>
PPD_DEV void move_plane(const KvEvictParams &p, const KvPlane &pl, const int32_t *kept, uint32_t u, int c0, int c1, int i0, int i1, int tid)
{
    switch (pl.unit) {
    case 16: move_rows<16, THREADS>(p, pl, kept, u, c0, c1, i0, i1, tid); break;
    case 8: move_rows<8, THREADS>(p, pl, kept, u, c0, c1, i0, i1, tid); break;
    case 4: move_rows<4, THREADS>(p, pl, kept, u, c0, c1, i0, i1, tid); break;
    case 2: move_rows<2, THREADS>(p, pl, kept, u, c0, c1, i0, i1, tid); break;
    default: move_rows<1, THREADS>(p, pl, kept, u, c0, c1, i0, i1, tid); break;
    }
}

// A slice's blocks: those of each plane in turn, each a range of rows (to another cache) or
// of columns (in place).
__global__ void __launch_bounds__(kMoveThreads) kv_move_kernel(const KvEvictParams p)
{
    pdl_release();
    pdl_wait();
    const uint32_t u = blockIdx.x / (uint32_t)p.move_blocks;
    int part = (int)(blockIdx.x % p.move_blocks), x = 0;
    while (part >= p.plane[x].parts) part -= p.plane[x++].parts;
    const KvPlane &pl = p.plane[x];
    const int b = (int)(u / (uint32_t)p.H % (uint32_t)p.B);
    const int len = ld_input(p.length + b);
    if (len < 0 || len > p.S_max) return;
    const int n = min(len, p.budget);
    if (pl.src == pl.dst && len <= p.budget) return;   // every row is in its place
    const int32_t *kept = p.kept + (size_t)u * p.budget;
    const int per_row = pl.row_bytes / pl.unit;
    int c0 = 0, c1 = per_row, i0 = 0, i1 = n;
    if (pl.src == pl.dst) {
        c0 = per_row * part / pl.parts;
        c1 = per_row * (part + 1) / pl.parts;
    } else {
        i0 = (int)((long long)p.budget * part / pl.parts);
        i1 = min(n, (int)((long long)p.budget * (part + 1) / pl.parts));
    }
    move_plane<kMoveThreads>(p, pl, kept, u, c0, c1, i0, i1, (int)threadIdx.x);
}

// Short caches: a warp a slice.  A lane holds four rows' ranks and counts, for each, the rows that
// come before it in order of weight; then the warp moves its planes' rows.
constexpr int kShortRows = 128;
__global__ void __launch_bounds__(128) kv_evict_short_kernel(const KvEvictParams p)
{
    __shared__ int32_t kept_s[4][kShortRows];
    pdl_release();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t u = blockIdx.x * 4 + warp;
    if (u >= p.slices) return;
    const int b = (int)(u / (uint32_t)p.H % (uint32_t)p.B);
    const int len = ld_input(p.length + b);
    const bool bad = len < 0 || len > p.S_max;
    if (u / p.H < p.B && u % p.H == 0 && lane == 0) {
        p.dev_status[b] = bad ? kErrCapacity : kOk;
        p.new_len[b] = bad ? len : min(len, p.budget);
    }
    const float *w = p.weight + (size_t)u * p.S_max;
    int32_t *kept = p.kept + (size_t)u * p.budget;
    constexpr int PER = kShortRows / 32;
    uint32_t r[PER];
    int before[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int j = lane + 32 * k;
        const bool in = !bad && j < len;
        r[k] = !in ? 0u : j < p.sink || j >= len - p.recent ? 0xFFFFFFFFu : weight_rank(ld_input(w + j));
        before[k] = in ? 0 : kShortRows;   // rows past the length are not kept
    }
    if (!bad && len > p.budget) {
#pragma unroll
        for (int k = 0; k < PER; ++k)
            for (int i = 0; i < min(32, len - 32 * k); ++i) {
                const uint32_t x = __shfl_sync(0xffffffffu, r[k], i);
#pragma unroll
                for (int m = 0; m < PER; ++m) before[m] += x > r[m] || (x == r[m] && 32 * k + i < lane + 32 * m);
            }
    }
    int n = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const bool take = before[k] < p.budget && lane + 32 * k < len;
        const uint32_t all = __ballot_sync(0xffffffffu, take);
        if (take) {
            const int i = n + __popc(all & ((1u << lane) - 1u));
            kept_s[warp][i] = lane + 32 * k;
            kept[i] = lane + 32 * k;
        }
        n += __popc(all);
    }
    for (int i = n + lane; i < p.budget; i += 32) kept[i] = -1;
    if (bad) return;
    __syncwarp();
    for (int x = 0; x < p.planes; ++x) {
        const KvPlane &pl = p.plane[x];
        if (pl.src == pl.dst && len <= p.budget) continue;   // every row is in its place
        // a row of up to 1024 bytes in pieces that a step holds
        const int per_row = pl.row_bytes / pl.unit, most = 32 * kMoveDeep;
        for (int c = 0; c < per_row; c += most) move_plane<32>(p, pl, kept_s[warp], u, c, min(per_row, c + most), 0, n, lane);
        __syncwarp();
    }
}

cudaError_t launch_kv_evict(const KvEvictParams &p, cudaStream_t stream)
{
    // (a warp a slice / a block a slice, then the moves: 8.7 / 11 us for 128 slices of 31 rows, 22 / 28 us for
    // 640 of 128, but 20 / 9 us for 32 of 128)
    if (p.S_max <= kShortRows && p.slices >= 4ll * p.S_max)
        return launch_chained(kv_evict_short_kernel, dim3((unsigned)((p.slices + 3) / 4)), dim3(128), dim3(1), stream, p);
    // ranks in shared memory up to 40,000 rows (160 KB); read again instead, 32 slices of 16,384 rows
    // take 49 us in place of 25, 512 slices 174 in place of 163
    constexpr uint32_t most = 40000;
    static std::atomic<uint64_t> configured{0};
    cudaError_t e;
    if ((uint32_t)p.S_max <= most) {
        e = allow_smem(kv_select_kernel<true>, most * 4, configured);
        if (e == cudaSuccess)
            e = launch_chained_smem(kv_select_kernel<true>, dim3((unsigned)p.slices), dim3(kSelThreads), dim3(1), (uint32_t)p.S_max * 4u, stream, p);
    } else {
        e = launch_chained(kv_select_kernel<false>, dim3((unsigned)p.slices), dim3(kSelThreads), dim3(1), stream, p);
    }
    if (e != cudaSuccess) return e;
    return launch_chained(kv_move_kernel, dim3((unsigned)(p.slices * p.move_blocks)), dim3(kMoveThreads), dim3(1), stream, p);
}

}  // namespace ppd
