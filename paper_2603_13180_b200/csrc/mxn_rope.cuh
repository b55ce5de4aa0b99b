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
    float2 c[4], s[4];
};

__device__ __forceinline__ void load_turn(Turn& t, const float* row, int sub, int rot)
{
    const float4* c = reinterpret_cast<const float4*>(row + 8 * sub);
    const float4* s = reinterpret_cast<const float4*>(row + rot / 2 + 8 * sub);
    *reinterpret_cast<float4*>(t.c) = __ldg(c);
    *reinterpret_cast<float4*>(t.c + 2) = __ldg(c + 1);
    *reinterpret_cast<float4*>(t.s) = __ldg(s);
    *reinterpret_cast<float4*>(t.s + 2) = __ldg(s + 1);
}

// The lane's 16 elements as binary32 pairs for packed arithmetic: a[i] = first members 2i, 2i + 1 of the pairs that turn
// together, b[i] = their second members, for either order of the elements in memory (halves: the lane's two runs; pairs: the even
// and the odd elements of both).  Lanes that do not turn use the same arrangement.
struct Lane16 {
    float2 a[4], b[4];
};

template <bool PAIRS>
__device__ __forceinline__ void unpack(Lane16& x, const uint4* w)
{
    const uint32_t u[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (PAIRS) {
            x.a[i] = make_float2(bf16_lo(u[2 * i]), bf16_lo(u[2 * i + 1]));
            x.b[i] = make_float2(bf16_hi(u[2 * i]), bf16_hi(u[2 * i + 1]));
        } else {
            x.a[i] = make_float2(bf16_lo(u[i]), bf16_hi(u[i]));
            x.b[i] = make_float2(bf16_lo(u[4 + i]), bf16_hi(u[4 + i]));
        }
    }
}

// (a, b) -> (a cos - b sin, b cos + a sin), or the opposite angle (BACK: the transposed rotation, for the gradient).  FUSED: a
// product and a sum in one rounding; else every product and sum is one IEEE binary32 operation.
template <bool BACK, bool FUSED>
__device__ __forceinline__ void apply_turn(Lane16& x, const Turn& t)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 a = x.a[i], b = x.b[i], s = BACK ? make_float2(-t.s[i].x, -t.s[i].y) : t.s[i], m = make_float2(-s.x, -s.y);
        if (FUSED) {
            x.a[i] = __ffma2_rn(b, m, __fmul2_rn(a, t.c[i]));
            x.b[i] = __ffma2_rn(a, s, __fmul2_rn(b, t.c[i]));
        } else {
            // one by one: the compiler joins a packed product and a packed sum to one rounding
            const float2 c = t.c[i];
            x.a[i] = make_float2(__fadd_rn(__fmul_rn(a.x, c.x), __fmul_rn(b.x, m.x)), __fadd_rn(__fmul_rn(a.y, c.y), __fmul_rn(b.y, m.y)));
            x.b[i] = make_float2(__fadd_rn(__fmul_rn(b.x, c.x), __fmul_rn(a.x, s.x)), __fadd_rn(__fmul_rn(b.y, c.y), __fmul_rn(a.y, s.y)));
        }
    }
}

// lanes that hold one head: dim / 16, rounded up to a power of two
__host__ __device__ constexpr int lanes_per_head(int dim) { return dim <= 16 ? 1 : dim <= 32 ? 2 : dim <= 64 ? 4 : dim <= 128 ? 8 : 16; }

}  // namespace mxn
