// Position rotation shared by the per-head norm and the cache append: how a lane's elements pair up, and the turn itself.
//
// A head of `dim` elements is held by dim/16 lanes, two runs of eight elements each.  With rot rotated elements
//   halves: element i < rot/2 turns with element i + rot/2;   pairs: element 2i turns with element 2i + 1,
// by the angle whose cosine and sine stand at [i] and [rot/2 + i] of the token's table row.  Lane `sub` < rot/16 holds the
// pairs i = 8*sub .. 8*sub+7 in either order; the lanes behind them hold 16 consecutive elements that are only passed on.
// Both members of a pair are in one lane, so the rotation needs no exchange between lanes, and a lane's eight cosines and
// sines are 32 consecutive bytes each.
#pragma once

#include "mxn_device.cuh"

namespace mxn {

struct LanePairs {
    int o0, o1;   // element offsets of the lane's two runs of eight
    bool turns;
};

__device__ __forceinline__ LanePairs lane_pairs(int sub, int rot, bool pairs)
{
    LanePairs p;
    p.turns = 16 * sub < rot;
    const bool halves = p.turns && !pairs;
    p.o0 = halves ? 8 * sub : 16 * sub;
    p.o1 = halves ? rot / 2 + 8 * sub : 16 * sub + 8;
    return p;
}

struct Turn {
    float c[8], s[8];
};

__device__ __forceinline__ void load_turn(Turn& t, const float* row, int sub, int rot)
{
    const float4* c = reinterpret_cast<const float4*>(row + 8 * sub);
    const float4* s = reinterpret_cast<const float4*>(row + rot / 2 + 8 * sub);
    *reinterpret_cast<float4*>(t.c) = __ldg(c);
    *reinterpret_cast<float4*>(t.c + 4) = __ldg(c + 1);
    *reinterpret_cast<float4*>(t.s) = __ldg(s);
    *reinterpret_cast<float4*>(t.s + 4) = __ldg(s + 1);
}

// x[0..7], x[8..15]: the lane's two runs.  Every product and sum is one IEEE binary32 operation.  BACK turns by the
// opposite angle (the transposed rotation, for the gradient).
template <bool PAIRS, bool BACK>
__device__ __forceinline__ void apply_turn(float* x, const Turn& t)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int ia = PAIRS ? 2 * i : i, ib = PAIRS ? 2 * i + 1 : i + 8;
        const float a = x[ia], b = x[ib], c = t.c[i], s = BACK ? -t.s[i] : t.s[i];
        x[ia] = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
        x[ib] = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
    }
}

__device__ __forceinline__ void unpack8(float* x, uint4 w)
{
    x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
    x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
}

// lanes that hold one head: dim / 16, rounded up to a power of two
__host__ __device__ constexpr int lanes_per_head(int dim) { return dim <= 16 ? 1 : dim <= 32 ? 2 : dim <= 64 ? 4 : dim <= 128 ? 8 : 16; }

}  // namespace mxn
