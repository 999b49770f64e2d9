// ppd_pages.cu -- a pool of pages shared by sequences: pages for the rows that sequences
// gain and back from the rows that they lose (ppd_page_assign), and rows of K and V into
// their slots (ppd_page_append).
#include "ppd_device.cuh"
#include "ppd_kernels.h"

namespace ppd {

// ------------------------------------------------------------------ pages

// held = ceil(old / page), want = ceil(new / page).  With S the stack of free pages and R the
// pages given back, in order of sequence and index, the call takes the last K entries of S
// followed by R, in that order, for the K pages that are needed: entry i of those is either
// an entry of S or a released one, so nothing is pushed before it is popped, and a call with
// lengths exchanged restores the pool.
//
// One grid and no scratch: every CTA scans the lengths itself (B of them, a few kilobytes out of
// L2) and then does its share of three lists, each found by bisection of the scan's sums in
// shared memory: slots, table entries taken, stack entries pushed.  What a CTA writes (entries
// from `held` on, stack entries past those that are read) none reads, and what all read at the
// start (lengths, n_free) none writes.
constexpr int kAssignThreads = 512, kAssignWarps = kAssignThreads / 32;

struct Sums3 {
    long long a, b, c;
};

// Exclusive sums over the block's threads; `total` those of all.
PPD_DEV Sums3 block_sums(Sums3 v, Sums3 *s_warp, Sums3 &total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Sums3 x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long a = __shfl_up_sync(0xffffffffu, x.a, o), b = __shfl_up_sync(0xffffffffu, x.b, o), c = __shfl_up_sync(0xffffffffu, x.c, o);
        if (lane >= o) x.a += a, x.b += b, x.c += c;
    }
    __syncthreads();   // an earlier call's readers are done
    if (lane == 31) s_warp[warp] = x;
    __syncthreads();
    Sums3 before{0, 0, 0};
    total = before;
    for (int w = 0; w < kAssignWarps; ++w) {
        const Sums3 y = s_warp[w];
        if (w < warp) before.a += y.a, before.b += y.b, before.c += y.c;
        total.a += y.a, total.b += y.b, total.c += y.c;
    }
    return Sums3{before.a + x.a - v.a, before.b + x.b - v.b, before.c + x.c - v.c};
}

// The sequence whose part of the sums holds i: the last b with sum[b] <= i (i < sum[B]).
PPD_DEV int find_part(const int *sum, int B, int i)
{
    int lo = 0, hi = B;   // sum[lo] <= i < sum[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sum[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kAssignThreads) page_assign_kernel(const PageAssignParams p)
{
    extern __shared__ int sums[];   // [B + 1] of each: pages released, taken; slots
    __shared__ Sums3 s_warp[kAssignWarps];
    int *rel = sums, *tk = sums + p.B + 1, *sl = tk + p.B + 1;
    const int tid = threadIdx.x, B = p.B, sh = p.page_shift;
    pdl_wait();
    pdl_release();

    // ---- this thread's sequences [b0, b1): what they release and need
    const int each = (B + kAssignThreads - 1) / kAssignThreads;
    const int b0 = min(B, tid * each), b1 = min(B, b0 + each);
    const int limit = p.max_pages << sh;
    const int n_free = min(max(ld_input(p.n_free), 0), p.n_pages);
    auto pages_of = [&](int rows) { return (int)(((long long)rows + (1 << sh) - 1) >> sh); };
    struct Need {
        int old_len, new_len, release, take, rows;
        bool valid;
    };
    auto need_of = [&](int b) {
        Need x{ld_input(p.old_len + b), ld_input(p.new_len + b), 0, 0, 0, false};
        x.valid = x.old_len >= 0 && x.old_len <= limit && x.new_len >= 0 && x.new_len <= limit;
        if (x.valid) {
            const int d = pages_of(x.new_len) - pages_of(x.old_len);
            x.take = max(d, 0);
            x.release = max(-d, 0);
            x.rows = max(x.new_len - x.old_len, 0);
        }
        return x;
    };
    Sums3 mine{0, 0, 0}, total;
    for (int b = b0; b < b1; ++b) {
        const Need x = need_of(b);
        mine.a += x.release, mine.b += x.take, mine.c += x.rows;
    }
    Sums3 at = block_sums(mine, s_warp, total);
    const long long R = total.a, available = n_free + R;

    // ---- served in order while the pages, and the slots, last
    auto served = [&](const Need &x, const Sums3 &upto) {
        return x.valid && (x.take == 0 || upto.b <= available) && (x.rows == 0 || upto.c <= p.max_slots);
    };
    Sums3 upto = at;
    mine = Sums3{0, 0, 0};
    for (int b = b0; b < b1; ++b) {
        const Need x = need_of(b);
        upto.b += x.take, upto.c += x.rows;
        if (served(x, upto)) mine.a += x.release, mine.b += x.take, mine.c += x.rows;
    }
    Sums3 part = block_sums(mine, s_warp, total);   // (releases are served always)
    upto = at;
    for (int b = b0; b < b1; ++b) {
        const Need x = need_of(b);
        upto.b += x.take, upto.c += x.rows;
        const bool ok = served(x, upto);
        rel[b] = (int)part.a, tk[b] = (int)part.b, sl[b] = (int)part.c;
        if (blockIdx.x == 0) {
            p.slot_start[b] = (int)part.c;
            p.out_len[b] = ok ? x.new_len : x.old_len;
            p.dev_status[b] = ok ? kOk : kErrCapacity;
        }
        if (ok) part.a += x.release, part.b += x.take, part.c += x.rows;
    }
    const int n_rel = (int)min(R, (long long)INT32_MAX), n_tk = (int)total.b, n_sl = (int)total.c;
    const long long left = available - n_tk;   // entries of S and R that stay
    if (tid == 0) {
        rel[B] = n_rel, tk[B] = n_tk, sl[B] = n_sl;
        if (blockIdx.x == 0) {
            p.slot_start[B] = n_sl;
            *p.new_n_free = (int)min(left, (long long)p.n_pages);
        }
    }
    __syncthreads();

    auto released = [&](int i) {
        const int b = find_part(rel, B, i);
        return ld_input(p.table + (size_t)b * p.max_pages + pages_of(ld_input(p.new_len + b)) + (i - rel[b]));
    };
    auto taken = [&](int i) {
        const long long at = left + i;
        return at < n_free ? ld_input(p.free_pages + at) : released((int)(at - n_free));
    };
    // (unsigned: a step past the last of 2^31 entries does not turn negative)
    const unsigned first = blockIdx.x * kAssignThreads + tid, step = gridDim.x * kAssignThreads;

    // ---- slots, four at a time
    for (unsigned at4 = 4 * first; at4 < (unsigned)n_sl; at4 += 4 * step) {
        const int i0 = (int)at4;
        int b = find_part(sl, B, i0), b_end = sl[b + 1];
        int old_len = ld_input(p.old_len + b), held = pages_of(old_len);
        int last = -1, page = 0;
        int v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = i0 + e;
            v[e] = 0;
            if (i >= n_sl) break;
            if (i >= b_end) {
                do ++b;
                while (sl[b + 1] <= i);
                b_end = sl[b + 1];
                old_len = ld_input(p.old_len + b);
                held = pages_of(old_len);
                last = -1;
            }
            const int pos = old_len + (i - sl[b]), idx = pos >> sh;
            if (idx != last) {
                page = idx < held ? ld_input(p.table + (size_t)b * p.max_pages + idx) : taken(tk[b] + idx - held);
                last = idx;
            }
            v[e] = (page << sh) + (pos & ((1 << sh) - 1));
        }
        if (p.vec && i0 + 4 <= n_sl) {
            *reinterpret_cast<int4 *>(p.slots + i0) = make_int4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i0 + e < n_sl) p.slots[i0 + e] = v[e];
        }
    }
    // ---- pages taken into the tables
    for (unsigned i = first; i < (unsigned)n_tk; i += step) {
        const int b = find_part(tk, B, (int)i);
        p.table[(size_t)b * p.max_pages + pages_of(ld_input(p.old_len + b)) + ((int)i - tk[b])] = taken((int)i);
    }
    // ---- pages released and not taken onto the stack
    const int n_push = (int)max(0ll, min(left - n_free, (long long)(p.n_pages - n_free)));
    for (unsigned i = first; i < (unsigned)n_push; i += step) p.free_pages[n_free + i] = released((int)i);
}

cudaError_t launch_page_assign(const PageAssignParams &p, int num_sms, cudaStream_t stream)
{
    static std::atomic<uint64_t> configured{0};
    const uint32_t smem = 3u * (uint32_t)(p.B + 1) * 4u;
    const cudaError_t e = allow_smem(page_assign_kernel, 3u * (kMaxAssign + 1) * 4u, configured);
    if (e != cudaSuccess) return e;
    // a CTA an SM at most, and one where a few thousand slots are all there can be
    const long long want = ((long long)p.max_slots + 4 * kAssignThreads - 1) / (4 * kAssignThreads);
    const int grid = (int)(want < num_sms ? (want > 0 ? want : 1) : num_sms);
    return launch_chained_smem(page_assign_kernel, dim3((unsigned)grid), dim3(kAssignThreads), dim3(1), smem, stream, p);
}

// ------------------------------------------------------------------ rows into pages

// A block takes kAppendRows rows of a slice, K and V; 16 bytes of a pool's row a thread and
// step, kInFlight steps' loads in flight.  HBM for prompts; for paths the rounds of blocks, most of whose threads
// have nothing to do (2048 blocks of up to six rows 6.0 us; 576, one round, 3.1; one 2.6).
constexpr int kAppendRows = 64, kAppendThreads = 256, kInFlight = 4;

template <bool F32>
__global__ void __launch_bounds__(kAppendThreads) page_append_kernel(const PageAppendParams p)
{
    pdl_wait();
    pdl_release();
    const int per_row = p.D / 8;
    const long long slice = blockIdx.x / p.chunks;
    const int j0 = (int)(blockIdx.x - slice * p.chunks) * kAppendRows;
    const int h = (int)(slice % p.H), b = (int)(slice / p.H % p.B), l = (int)(slice / ((long long)p.H * p.B));
    const int s0 = ld_input(p.slot_start + b), s1 = ld_input(p.slot_start + b + 1);
    const bool bad = s0 < 0 || s1 < s0 || s1 > p.max_slots || s1 - s0 > p.T;
    if (l == 0 && h == 0 && j0 == 0 && threadIdx.x == 0) p.dev_status[b] = bad ? kErrCapacity : kOk;
    if (bad) return;
    const int n = min(kAppendRows, s1 - s0 - j0) * per_row;
    const long long pool_rows = (long long)p.n_pages << p.page_shift;
    for (int w0 = threadIdx.x; w0 < n; w0 += kInFlight * kAppendThreads) {
        long long to[kInFlight];
        uint4 k[kInFlight], v[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const int w = w0 + u * kAppendThreads;
            to[u] = -1;
            if (w >= n) continue;
            const int j = j0 + w / per_row, c = w % per_row;
            const int slot = ld_input(p.slots + s0 + j);
            const int row = p.rows ? ld_input(p.rows + (size_t)b * p.T + j) : j;
            if (slot < 0 || slot >= pool_rows || row < 0 || row >= p.T) continue;
            const long long page = slot >> p.page_shift, at = slot & ((1 << p.page_shift) - 1);
            to[u] = (((((long long)l * p.n_pages + page) * p.H + h) << p.page_shift) + at) * per_row + c;
            const size_t from = ((size_t)slice * p.T + row) * per_row + c;
            if (F32) {
                const float4 *kf = reinterpret_cast<const float4 *>(p.k_new) + 2 * from, *vf = reinterpret_cast<const float4 *>(p.v_new) + 2 * from;
                const float4 a = ld_input(kf), d = ld_input(kf + 1), e = ld_input(vf), f = ld_input(vf + 1);
                k[u] = make_uint4(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w), pack_bf16(d.x, d.y), pack_bf16(d.z, d.w));
                v[u] = make_uint4(pack_bf16(e.x, e.y), pack_bf16(e.z, e.w), pack_bf16(f.x, f.y), pack_bf16(f.z, f.w));
            } else {
                k[u] = ld_input(reinterpret_cast<const uint4 *>(p.k_new) + from);
                v[u] = ld_input(reinterpret_cast<const uint4 *>(p.v_new) + from);
            }
        }
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            if (to[u] < 0) continue;
            reinterpret_cast<uint4 *>(p.k_pages)[to[u]] = k[u];
            reinterpret_cast<uint4 *>(p.v_pages)[to[u]] = v[u];
        }
    }
}

cudaError_t launch_page_append(PageAppendParams p, cudaStream_t stream)
{
    p.chunks = (p.T + kAppendRows - 1) / kAppendRows;
    const dim3 grid((unsigned)(p.slices * p.chunks));
    return p.f32 ? launch_chained(page_append_kernel<true>, grid, dim3(kAppendThreads), dim3(1), stream, p)
                 : launch_chained(page_append_kernel<false>, grid, dim3(kAppendThreads), dim3(1), stream, p);
}

int page_append_chunks(int T) { return (T + kAppendRows - 1) / kAppendRows; }

}  // namespace ppd
