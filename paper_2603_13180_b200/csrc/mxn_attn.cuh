// Declarations shared by the two attention kernels over the 8-bit cache.
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>

#include "mxn_async.cuh"
#include "mxn_device.cuh"
#include "mxn_internal.h"

namespace mxn {

struct AttnMaps {
    CUtensorMap k, v;   // codes as [pages * heads, page, dim] bytes
};

// tensor map of the queries in boxes of 64 dimensions of `heads` heads of `tokens` tokens, 128-byte swizzle
bool make_query_map(CUtensorMap* map, const AttnParams& P, int heads, int tokens);
// the kernel for many query rows (mxn_prompt.cu)
cudaError_t launch_prompt(const AttnParams& P, const AttnMaps& M, int64_t ctas, cudaStream_t stream);
cudaError_t read_prompt_counters(unsigned int* timeouts, unsigned int* bad);
cudaError_t reset_prompt_counters(bool timeouts);

// A sequence's rows and places.  The last query stands at the sequence's last token, however many of the rows or of the keys the
// call's bounds let through: places go by the lists as they stand, the bounds only cut what is computed and read.
struct AttnSequence {
    int q0, nq;    // first row, rows computed (0 where the list of rows is no rising one)
    int shift;     // place of the first query
    int len;       // keys that may be read
};
__device__ __forceinline__ AttnSequence attn_sequence(const AttnParams& P, int seq)
{
    AttnSequence s;
    s.q0 = __ldg(P.cu_q + seq);
    const int end = __ldg(P.cu_q + seq + 1), all = max(0, __ldg(P.lens + seq));
    s.nq = s.q0 < 0 || end <= s.q0 ? 0 : max(0, min(min(end, (int)P.n) - s.q0, P.max_q));
    s.shift = s.nq > 0 ? all - (end - s.q0) : 0;
    s.len = min(all, P.max_len);
    return s;
}
// first key that a query at `pos` sees.  The place may lie before the first token and the window be any up to 2^31 - 1, so the
// difference takes more than 32 bits.
__device__ __forceinline__ int first_seen(int pos, int window)
{
    return window > 0 ? (int)max((int64_t)0, (int64_t)pos - window + 1) : 0;
}

// What a row may see, apart from its sequence's length: kCausal (places up to its own, from the window's start on), kSinks (the same, and
// the first tokens), kTree (all in front of the sequence's new tokens, and those of these whose bits its row of the mask has)
enum { kCausal = 0, kSinks = 1, kTree = 2 };

// The keys of a call as a list of whole tiles of T tokens: with kSinks those of the first tokens, then those from the window on.
struct KeyList {
    int head, gap;   // tokens in front of the gap (whole tiles), tokens that the gap leaves out
    __device__ __forceinline__ int at(int u) const { return u < head ? u : u + gap; }
};
template <int T>
__device__ __forceinline__ KeyList key_list(int sinks, int lo)   // lo: the window's first tile
{
    KeyList k;
    k.head = (int)min((int64_t)lo, ((int64_t)sinks + T - 1) / T * T);
    k.gap = lo - k.head;
    return k;
}
// 32 bits from bit d of a row of the mask on; all that stands in front of it is seen
__device__ __forceinline__ uint32_t tree_bits(const uint32_t* row, int words, int64_t d)
{
    if (d <= -32) return 0xFFFFFFFFu;
    if (d < 0) return (__ldg(row) << (int)-d) | ((1u << (int)-d) - 1u);
    const int64_t w = d >> 5;
    return __funnelshift_r(w < words ? __ldg(row + w) : 0u, w + 1 < words ? __ldg(row + w + 1) : 0u, (uint32_t)d & 31u);
}

// tiled copy of a box of codes (no multicast); x = 0, y = first token within its page, z = page * heads + head
__device__ __forceinline__ void tma_load_codes(uint32_t dst, const CUtensorMap* map, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 :: "r"(dst), "l"(map), "r"(0), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// The softmax's sum and its range.  While the value scales lie within kApart binades of c0, the sum is in units of 2^(R - 1 - c0): its
// terms are the weights times 2^(c0 - sv).  R follows the largest s + sv to within 54, so the largest score's term lies between 2^-16
// and 2^71, and a step of R that is too large for binary32 (the sum so far becomes 0) only drops terms below 2^-39 of it.  A tile whose
// scales lie farther away (a run of zero values has scale 2^-127) is summed apart: with exponentials of its own, terms 2^(s - r), and a
// reference r of the sum that follows the scores alone, raised where a score lies kLift above it.
constexpr float kApart = 16.0f, kLift = 60.0f;
// v 2^d for a whole d whose power may lie outside binary32's range where the product does not
__device__ __forceinline__ float times_pow2(float v, float d)
{
    const float h = floorf(0.5f * d);
    return v * ex2(h) * ex2(d - h);
}
// a product of 16 x 16 by 16 x 8, binary32 sums
__device__ __forceinline__ void mma_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the four E4M3 codes of a word -> two f16 pairs
__device__ __forceinline__ void widen(uint32_t w, uint32_t& lo, uint32_t& hi)
{
    asm("{ .reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h; }" : "=r"(lo), "=r"(hi) : "r"(w));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// 2^(byte - 127), the value of an E8M0 byte
__device__ __forceinline__ float e8m0_to_f32(uint32_t b) { return __uint_as_float(b == 0 ? 0x00400000u : b << 23); }

}  // namespace mxn
