// Declarations shared by the two attention kernels over the 8-bit cache.
#pragma once

#include <cuda.h>

#include "mxn_async.cuh"
#include "mxn_device.cuh"
#include "mxn_internal.h"

namespace mxn {

struct AttnMaps {
    CUtensorMap k, v;   // codes as [pages * heads, page, dim] bytes
};

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
// 2^(byte - 127), the value of an E8M0 byte
__device__ __forceinline__ float e8m0_to_f32(uint32_t b) { return __uint_as_float(b == 0 ? 0x00400000u : b << 23); }

}  // namespace mxn
