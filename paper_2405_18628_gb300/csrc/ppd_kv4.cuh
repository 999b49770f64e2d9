// ppd_kv4.cuh -- the 4-bit cache format, and what the kernels that read it share.
//
// A row of D channels is D / 2 bytes of codes and one scale byte for each 32 channels.
// A 32-bit word holds eight channels: nibble p is channel 2 (p % 4) + p / 4, so that one
// mask takes a pair of neighbouring channels out of a word into the halves of a register.
// A code c stands for s (c - 8), a scale byte b for s = (1 + (b % 8) / 8) 2^(b / 8 - 20).
// s has four significant bits and c - 8 at most three, so that every value is a bf16
// number: the tensor cores multiply exactly what the cache holds.
#pragma once

#include "ppd_device.cuh"

#include <cuda_bf16.h>
#include <cstdint>

namespace ppd {

constexpr int kKv4Group = 32;   // channels of a scale

PPD_DEV uint32_t bf16x2_fma(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}

// A scale as fp32.  The byte's exponent field counts from 2^-20, fp32's from 2^-127.
PPD_DEV float kv4_scale(uint32_t b) { return __uint_as_float((b + 856u) << 20); }

// Codes become bf16 values without a conversion: bits 0..7 of a bf16 number alone (seven of
// the mantissa, the lowest of the exponent) stand for that byte times 2^-133, so a masked code in
// bits 0..3 is c 2^-133 and one in bits 4..7 is 16 c 2^-133, where it lies.  One fused multiply-add
// with 2^113 s (or a sixteenth of it) and -8 s 2^-20 then makes kKv4Unit s (c - 8): exact, and a
// word of eight codes takes one shift instead of three.  What the unit leaves over is a power
// of two: the softmax scale takes up K's, the outputs V's.
constexpr float kKv4Unit = 1.f / (1 << 20), kKv4Shift = 20.f;
constexpr int kKv4UnitLog2 = -20;
struct Kv4Scale {
    uint32_t s, s16, off;   // of a pair of codes, each
};
// `two` holds one scale byte in bits 0..7 and one in bits 16..23.
PPD_DEV Kv4Scale kv4_scales(uint32_t two)
{
    Kv4Scale r;
    r.s = (two + 0x06E006E0u) << 4;             // 2^113 s as bf16 bits
    r.s16 = r.s - 0x02000200u;
    r.off = bf16x2_fma(r.s, 0x80088008u, 0x80008000u);   // times -2^-130
    return r;
}
// kKv4Unit times the values of the pairs of codes in bits 0..3 and 16..19, and in 4..7 and 20..23.
PPD_DEV uint32_t kv4_low(uint32_t w, const Kv4Scale &k) { return bf16x2_fma(w & 0x000F000Fu, k.s, k.off); }
PPD_DEV uint32_t kv4_high(uint32_t w, const Kv4Scale &k) { return bf16x2_fma(w & 0x00F000F0u, k.s16, k.off); }
// The four pairs of a word: channels (0, 1), (2, 3), (4, 5), (6, 7).
PPD_DEV void kv4_word(uint32_t w, const Kv4Scale &k, uint32_t (&v)[4])
{
    v[0] = kv4_low(w, k);
    v[1] = kv4_high(w, k);
    v[2] = kv4_low(w >> 8, k);
    v[3] = kv4_high(w >> 8, k);
}
// A pair of such values without the unit.
PPD_DEV uint32_t kv4_whole(uint32_t v) { return bf16x2_fma(v, 0x49804980u, 0x80008000u); }

// Two fp32 values as a bf16 pair, the first in the low half.
PPD_DEV uint32_t bf16x2(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// The pair pp as bf16 hi + lo like split_bf16x2, the rounding done by packed fp32 operations:
// s = p + 2^16 p has 24 bits, so s - 2^16 p is p to eight.  (p below 2^111.)
PPD_DEV void split_bf16x2_fma(uint64_t pp, uint32_t &hi, uint32_t &lo)
{
    const uint64_t big = pack2(65536.f, 65536.f), neg = pack2(-65536.f, -65536.f), m1 = pack2(-1.f, -1.f);
    const uint64_t h = fma2(pp, neg, fma2(pp, big, pp));
    float h0, h1, l0, l1;
    unpack2(h, h0, h1);
    unpack2(fma2(h, m1, pp), l0, l1);
    hi = __byte_perm(__float_as_uint(h0), __float_as_uint(h1), 0x7632);
    lo = bf16x2(l0, l1);
}

// D += A B: A 16 x 16 rows of bf16, B 16 x 8, fp32 accumulators.
PPD_DEV void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// An 8 x 8 tile of 16-bit values, row lane / 4, columns 2 (lane % 4) and the next: transposed.
PPD_DEV uint32_t movmatrix(uint32_t x)
{
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
    return d;
}

// Asynchronous copies into shared memory; bytes beyond `n` of the 16 (or 4) read as zero.
PPD_DEV void cp_async16(uint32_t dst, const void *src, uint32_t n)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
PPD_DEV void cp_async4(uint32_t dst, const void *src, uint32_t n)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
PPD_DEV void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
PPD_DEV void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

PPD_DEV uint32_t ld_shared_u32(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
PPD_DEV uint32_t ld_shared_u8(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
PPD_DEV uint2 ld_shared_u64(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}
PPD_DEV uint4 ld_shared_u128(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}

// A warpgroup gives registers back, or takes up what others gave (a multiple of 8 a thread;
// all its warps execute it).
template <int N>
PPD_DEV void reg_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
PPD_DEV void reg_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

// Element i, i + 1 of a bf16 or fp32 tensor as a bf16 pair (fp32 rounded to nearest);
// i even.
PPD_DEV uint32_t ld_pair(const void *p, size_t i, bool f32)
{
    if (!f32) return (uint32_t)ld_input(reinterpret_cast<const int *>(p) + (i >> 1));
    const float *f = reinterpret_cast<const float *>(p) + i;
    return bf16x2(ld_input(f), ld_input(f + 1));
}

// What dev_status says of a sequence: a malformed tree, or a prefix outside the cache.
// Every lane of one warp gets the answer.
PPD_DEV int tree_status(const int32_t *parent, int T, int prefix, int S_max, int lane)
{
    bool bad = false;
    for (int i = lane; i < T; i += 32) {
        const int p = ld_input(parent + i);
        bad |= i == 0 ? p != -1 : (p < 0 || p >= i);
    }
    if (__any_sync(0xffffffffu, bad)) return kErrTree;
    return prefix < 0 || prefix > S_max ? kErrCapacity : kOk;
}

}  // namespace ppd
