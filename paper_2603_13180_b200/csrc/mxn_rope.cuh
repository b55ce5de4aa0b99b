// Position rotation shared by the per-head norm and the cache append: how a lane's elements pair up, and the turn itself.
//
// A head of `dim` elements is held by dim/16 lanes, two runs of eight elements each.  With rot rotated elements
//   halves: element i < rot/2 turns with element i + rot/2;   pairs: element 2i turns with element 2i + 1,
// by the angle whose cosine and sine stand at [i] and [rot/2 + i] of the token's table row.  Both members of a pair are in one lane,
// so the rotation needs no exchange between lanes.  Neighbouring lanes hold neighbouring runs, so that a load or store of one run
// by all of them touches whole 32-byte sectors (with 16 consecutive elements a lane, every sector was asked for twice: 16384 tokens
// of 32 heads of 64 in pairs, backward: 57 us, now 37).
//   halves: lane `sub` < rot/16 holds elements 8*sub .. 8*sub+7 and those rot/2 further on; the lanes behind them hold what is
//     not rotated, again in two runs;   pairs: 8*sub .. 8*sub+7 and those dim/2 further on, each run rotated or not by itself.
#pragma once

#include "mxn_device.cuh"

namespace mxn {

struct LanePairs {
    int o0, o1;            // element offsets of the lane's two runs of eight
    bool turns, turns1;    // whether they are rotated (the second only with the first)
};

__device__ __forceinline__ LanePairs lane_pairs(int sub, int dim, int rot, bool pairs)
{
    LanePairs p;
    p.turns = (pairs ? 8 : 16) * sub < rot;
    p.o0 = pairs || p.turns ? 8 * sub : 8 * sub + rot / 2;   // halves, not rotated: rot + 8 * (sub - rot / 16)
    p.o1 = p.o0 + (pairs ? dim / 2 : p.turns ? rot / 2 : (dim - rot) / 2);
    p.turns1 = pairs ? p.o1 < rot : p.turns;
    return p;
}

// for lanes that turn
struct Turn {
    float2 c[4], s[4];
};

template <bool PAIRS>
__device__ __forceinline__ void load_turn(Turn& t, const float* row, const LanePairs& lp, int rot)
{
    // the runs' first angles: four of each run, or eight of the first
    const float4* c0 = reinterpret_cast<const float4*>(row + (PAIRS ? lp.o0 / 2 : lp.o0));
    const float4* c1 = PAIRS ? reinterpret_cast<const float4*>(row + lp.o1 / 2) : c0 + 1;
    *reinterpret_cast<float4*>(t.c) = __ldg(c0);
    *reinterpret_cast<float4*>(t.s) = __ldg(c0 + rot / 8);
    if (!PAIRS || lp.turns1) {
        *reinterpret_cast<float4*>(t.c + 2) = __ldg(c1);
        *reinterpret_cast<float4*>(t.s + 2) = __ldg(c1 + rot / 8);
    }
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
template <bool BACK, bool FUSED, bool PAIRS>
__device__ __forceinline__ void apply_turn(Lane16& x, const Turn& t, const LanePairs& lp)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (PAIRS && i >= 2 && !lp.turns1) break;   // pairs: the second run
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
