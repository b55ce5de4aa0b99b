// RMS norm of every query and key head with the position rotation in the same pass, and its gradient.
//
//   n = x * r,  r = 1 / sqrt(mean x^2 + eps) over the head;  u = n * gamma;  y = R(position) u
//   du = R^T dy;  dgamma = sum over tokens and heads of du * n;  h = du * gamma;  dx = r * (h - n * mean(h * n))
//
// Both are bound by HBM: 4 bytes an element forward (read x, write y), 6 backward (x, dy, dx).  A head of `dim` elements is
// held by dim/16 lanes (see mxn_rope.cuh), so the head's sums take log2(dim/16) shuffles and the rotation none; a warp
// works on 32*16/dim heads at a time and keeps the token's cosines and sines in registers over all of its heads.
// The gradient recomputes r from x, which it reads anyway, instead of loading a saved one.
//
// Measured, 32 query and 8 key heads of 128 (on the device alone, in turn with other work in brackets): 16384 tokens forward 62 us (62),
// 5.4 TB/s; backward with both gains' gradients 90 us (91), 5.6 TB/s; 64 tokens 2.5 us and 5.1 us, the latency of a start and one (two)
// trips to memory.  4099 tokens of 32 and 4 heads of 64 in pairs, half of each rotated, backward: 15 us (18), 3.7 TB/s, of which 2.6 are
// the second launch that joins the gains' sums and some 3 the start.
#include <cuda_bf16.h>

#include "mxn_internal.h"
#include "mxn_rope.cuh"

namespace mxn {

namespace {

constexpr int kSMs = 148;   // B200
constexpr int kWarps = 4;   // per CTA

__device__ unsigned int g_heads_bad = 0;   // tokens whose position lies outside the table

__device__ __forceinline__ uint4 ld16(const uint16_t* p)
{
    uint4 r;   // through the coherent path: the output may be written in place
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
    return r;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
template <bool PAIRS>
__device__ __forceinline__ void store(uint16_t* p, int second, const Lane16& x)   // second: bytes to the second run
{
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (PAIRS) {
            r[2 * i] = pack2(x.a[i].x, x.b[i].x);
            r[2 * i + 1] = pack2(x.a[i].y, x.b[i].y);
        } else {
            r[i] = pack2(x.a[i].x, x.a[i].y);
            r[4 + i] = pack2(x.b[i].x, x.b[i].y);
        }
    }
    st_v4(p, r);
    st_v4(reinterpret_cast<char*>(p) + second, r + 4);
}
__device__ __forceinline__ void scale(Lane16& x, float r)
{
    const float2 f = make_float2(r, r);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x.a[i] = __fmul2_rn(x.a[i], f);
        x.b[i] = __fmul2_rn(x.b[i], f);
    }
}
__device__ __forceinline__ void scale(Lane16& x, const Lane16& g)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x.a[i] = __fmul2_rn(x.a[i], g.a[i]);
        x.b[i] = __fmul2_rn(x.b[i], g.b[i]);
    }
}
// sum of x y over the lane's elements
__device__ __forceinline__ float dot(const Lane16& x, const Lane16& y)
{
    float2 s = __fmul2_rn(x.a[0], y.a[0]), t = __fmul2_rn(x.b[0], y.b[0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) {
        s = __ffma2_rn(x.a[i], y.a[i], s);
        t = __ffma2_rn(x.b[i], y.b[i], t);
    }
    s = __fadd2_rn(s, t);
    return s.x + s.y;
}
__device__ __forceinline__ void fill(Lane16& x, float v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x.a[i] = x.b[i] = make_float2(v, v);
}
__device__ __forceinline__ void copy16(uint32_t dst, const char* src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t addr)
{
    uint4 r;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(addr) : "memory");
    return r;
}
template <int LP>
__device__ __forceinline__ float head_sum(float v)
{
#pragma unroll
    for (int o = LP / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
// mean x^2 + eps, and whether binary32 holds it and the squares with all of their digits
__device__ __forceinline__ float mean_square(float sum_sq, float inv_dim, float eps) { return fmaf(sum_sq, inv_dim, eps); }
__device__ __forceinline__ bool in_range(float ms) { return ms >= 0x1p-80f && ms <= 0x1p80f; }
// 1 / sqrt(mean x^2 + eps); 0 for a head of zeros without eps, which then stays zero
__device__ __forceinline__ float head_rcp(float ms) { return ms != 0.0f ? rsqrtf(ms) : 0.0f; }   // a NaN stays one
// The same for heads out of range (by a whole warp, whose other heads stay as they are): x is multiplied by a power of two, `unit`, first;
// the result is that of the new x, so that their product is x / rms all the same.
template <int LP>
__device__ __forceinline__ float head_rcp_any(Lane16& x, float ms, float inv_dim, float eps, float& unit)
{
    unit = ms > 0x1p80f ? 0x1p-80f : ms < 0x1p-80f ? 0x1p80f : 1.0f;
    scale(x, unit);
    return head_rcp(mean_square(head_sum<LP>(dot(x, x)), inv_dim, eps * unit * unit));
}

// a token's row of the rotation's table; rows and tokens are below 2^31
__device__ __forceinline__ int position(const HeadsParams& P, int64_t t) { return P.positions != nullptr ? __ldg(P.positions + t) : (int)t; }
// false: the position lies outside the table
template <bool PAIRS>
__device__ __forceinline__ bool turn_at(const HeadsParams& P, int pos, const LanePairs& lp, Turn& turn)
{
    if (pos < 0 || pos >= P.table_rows) return false;
    if (lp.turns) load_turn<PAIRS>(turn, P.cos_sin + (int64_t)pos * P.rot, lp, P.rot);
    return true;
}

// A warp takes U * G heads of one token, all of its loads at once.  `tight`: five CTAs an SM instead of four, for which the gain has to
// stay packed in its registers.  16384 tokens: 32 + 8 heads of 128 in pairs 63.9 -> 60.6 us, 16 + 2 heads of 256 64.8 -> 58.6, but 32 + 8
// heads of 128 in halves 64.7 -> 67.5.
__host__ __device__ constexpr bool tight(int lanes, bool pairs) { return pairs || lanes == 16; }
template <int LP, int U, bool PAIRS, bool NORM>
__global__ void __launch_bounds__(kWarps * 32, tight(LP, PAIRS) ? 5 : 1) rope_fwd_kernel(const HeadsParams P)
{
    constexpr int G = 32 / LP;   // heads a warp holds at a time
    pdl_prologue();
    const int lane = threadIdx.x & 31, sub = lane % LP, grp = lane / LP;
    const int64_t w = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const int64_t t = P.parts == 1 ? w : (int64_t)((uint64_t)w / (uint32_t)P.parts);
    if (t >= P.T) return;
    const int part = (int)(w - t * P.parts);
    const int heads = P.heads[0] + P.heads[1];
    const int h0 = part * U * G + grp;
    const bool live = 16 * sub < P.dim;
    const LanePairs lp = lane_pairs(live ? sub : 0, P.dim, P.rot, PAIRS);

    // head h of the two operands as one list
    const uint16_t* const xq = P.x[0] + t * P.x_stride[0];
    const uint16_t* const xk = P.x[1] + t * P.x_stride[1] - P.heads[0] * P.dim;
    uint16_t* const yq = P.y[0] + t * P.y_stride[0];
    uint16_t* const yk = P.y[1] + t * P.y_stride[1] - P.heads[0] * P.dim;
    uint4 raw[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = h0 + u * G;
        raw[u][0] = raw[u][1] = make_uint4(0u, 0u, 0u, 0u);
        if (live && h < heads) {
            const uint16_t* x = (h < P.heads[0] ? xq : xk) + h * P.dim;
            raw[u][0] = ld16(x + lp.o0);
            raw[u][1] = ld16(x + lp.o1);
        }
    }
    Turn turn;
    const bool good = P.cos_sin == nullptr || turn_at<PAIRS>(P, position(P, t), lp, turn);
    if (!good && lane == 0 && part == 0) atomicAdd(&g_heads_bad, 1u);
    uint4 gw[2];
    Lane16 g;
    int g_of = -1;   // whose gain they hold
    uint32_t later = 0;   // heads whose squares leave binary32's range: not written here
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int h = h0 + u * G;
        const int which = h >= P.heads[0];
        Lane16 x;
        unpack<PAIRS>(x, raw[u]);
        float r = 1.0f;
        if (NORM) {
            const float ms = mean_square(head_sum<LP>(dot(x, x)), P.inv_dim, P.eps);
            if (!in_range(ms) && h < heads) later |= 1u << u;
            r = head_rcp(ms);
            const uint16_t* gain = which ? P.gain[1] : P.gain[0];
            if (gain != nullptr && live) {
                if (g_of != which) {
                    gw[0] = __ldg(reinterpret_cast<const uint4*>(gain + lp.o0));
                    gw[1] = __ldg(reinterpret_cast<const uint4*>(gain + lp.o1));
                    if (!tight(LP, PAIRS)) unpack<PAIRS>(g, gw);
                    g_of = which;
                }
                if (tight(LP, PAIRS)) unpack<PAIRS>(g, gw);
                scale(x, g);
            }
        }
        if (P.cos_sin != nullptr) {
            if (!good) fill(x, __uint_as_float(0x7FC00000u));   // loud: no angle for this token
            else if (lp.turns) apply_turn<false, NORM, PAIRS>(x, turn, lp);
        }
        if (NORM) scale(x, r);   // the rotation leaves a common factor alone
        if (live && h < heads && !((later >> u) & 1u)) store<PAIRS>((which ? yk : yq) + h * P.dim + lp.o0, 2 * (lp.o1 - lp.o0), x);
    }
    if (NORM && __builtin_expect(__any_sync(0xFFFFFFFFu, later != 0u), 0)) {
        // once more from memory, which still holds them
#pragma unroll 1
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * G, which = h >= P.heads[0];
            const uint16_t* const in = (which ? xk : xq) + h * P.dim;
            const uint16_t* const gain = P.gain[which];
            const bool mine = live && h < heads && ((later >> u) & 1u);
            uint4 w[2] = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
            if (mine) {
                w[0] = ld16(in + lp.o0);
                w[1] = ld16(in + lp.o1);
            }
            Lane16 x;
            unpack<PAIRS>(x, w);
            float unit;
            const float r = head_rcp_any<LP>(x, mean_square(head_sum<LP>(dot(x, x)), P.inv_dim, P.eps), P.inv_dim, P.eps, unit);
            if (!mine) continue;
            if (gain != nullptr) {
                w[0] = __ldg(reinterpret_cast<const uint4*>(gain + lp.o0));
                w[1] = __ldg(reinterpret_cast<const uint4*>(gain + lp.o1));
                unpack<PAIRS>(g, w);
                scale(x, g);
            }
            if (P.cos_sin != nullptr) {
                if (!good) fill(x, __uint_as_float(0x7FC00000u));
                else if (lp.turns) apply_turn<false, NORM, PAIRS>(x, turn, lp);
            }
            scale(x, r);
            store<PAIRS>((which ? yk : yq) + h * P.dim + lp.o0, 2 * (lp.o1 - lp.o0), x);
        }
    }
}

// One CTA works for the queries or for the keys only (the CTAs are shared out by their head counts), so that a lane carries
// 16 sums of one gain's gradient.  A warp walks over a contiguous run of (token, group of heads) items, kRing - 1 of which are on
// their way to shared memory at a time (16-byte asynchronous copies; a thread reads back only what it asked for, so that nothing
// has to be synchronised): 4 KB in flight a warp against 2 KB that registers would hold (16384 tokens: registers 119 us, the ring 94).
// The row of the rotation's table that the next token needs is asked into L2 a token ahead (94 -> 89 us).
constexpr int kRing = 4;
template <int LP, bool PAIRS, bool NORM>
__global__ void __launch_bounds__(kWarps * 32, 4) rope_bwd_kernel(const HeadsParams P)
{
    constexpr int G = 32 / LP, N = NORM ? 4 : 2;        // 16-byte pieces of a thread's item
    constexpr uint32_t PIECE = kWarps * 32 * 16, SLOT = N * PIECE;
    __shared__ float sums[kWarps][256];
    __shared__ __align__(16) uint8_t ring[kRing * SLOT];
    pdl_prologue();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % LP, grp = lane / LP;
    const int which = (int)blockIdx.x >= P.ctas_q;
    const int64_t cta = which ? (int)blockIdx.x - P.ctas_q : (int)blockIdx.x, ctas = which ? (int)gridDim.x - P.ctas_q : P.ctas_q;
    const int heads = which ? P.heads[1] : P.heads[0], groups = (heads + G - 1) / G;
    const int64_t items = P.T * groups, warps = ctas * kWarps, w = cta * kWarps + warp;
    const int64_t begin = items * w / warps, end = items * (w + 1) / warps;
    const bool live = 16 * sub < P.dim;
    const int in_last = heads - (groups - 1) * G;       // heads of a token's last group
    const LanePairs lp = lane_pairs(live ? sub : 0, P.dim, P.rot, PAIRS);
    const int64_t first = groups > 0 ? begin / groups : 0;

    // byte addresses that run along with the walk: what is asked for (d: gradient, x: input) and what is written
    const int64_t d_stride = 2 * (which ? P.grad_stride[1] : P.grad_stride[0]), x_stride = 2 * (which ? P.x_stride[1] : P.x_stride[0]),
                  y_stride = 2 * (which ? P.y_stride[1] : P.y_stride[0]);
    const int step = 2 * G * P.dim, second = 2 * (lp.o1 - lp.o0);
    const int begin_group = (int)(begin - first * groups);
    const int64_t lane_at = 2 * ((int64_t)(begin_group * G + grp) * P.dim + lp.o0);
    const char* fd = reinterpret_cast<const char*>(which ? P.grad[1] : P.grad[0]) + first * d_stride + lane_at;
    const char* fx = reinterpret_cast<const char*>(which ? P.x[1] : P.x[0]) + first * x_stride + lane_at;
    char* y = reinterpret_cast<char*>(which ? P.y[1] : P.y[0]) + first * y_stride + lane_at;
    const int64_t token_bytes = (int64_t)groups * step;
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring) + threadIdx.x * 16;
    uint32_t f_at = ring_at, at = ring_at;
    int fg = begin_group, g = begin_group;
    int f_left = (int)(end - begin);   // a CTA for each kWarps items, or kSMs * 4 of them: far below 2^31
    auto fetch = [&]() {
        if (f_left > 0) {
            --f_left;
            const bool last = fg == groups - 1;
            const int bytes = live && (!last || grp < in_last) ? 16 : 0;   // 0: the piece is filled with zeros, nothing is read
            copy16(f_at, fd, bytes);
            copy16(f_at + PIECE, fd + second, bytes);
            if (NORM) {
                copy16(f_at + 2 * PIECE, fx, bytes);
                copy16(f_at + 3 * PIECE, fx + second, bytes);
            }
            f_at = f_at + SLOT == ring_at + kRing * SLOT ? ring_at : f_at + SLOT;
            fd += step;
            fx += step;
            ++fg;
            if (last) {
                fg = 0;
                fd += d_stride - token_bytes;
                fx += x_stride - token_bytes;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) fetch();

    Lane16 acc, gamma;
    fill(acc, 0.0f);
    fill(gamma, 1.0f);
    const uint16_t* const gain = which ? P.gain[1] : P.gain[0];
    if (NORM && gain != nullptr && live) {
        const uint4 u[2] = {__ldg(reinterpret_cast<const uint4*>(gain + lp.o0)), __ldg(reinterpret_cast<const uint4*>(gain + lp.o1))};
        unpack<PAIRS>(gamma, u);
    }
    Turn turn;
    // a lane's sum of squares from which on, or below which, a head may be out of range
    const float low = P.eps >= 0x1p-80f ? 0.0f : 0x1p-80f;
    bool good = true, fresh = true;
    int t = (int)first;
    // the token's row of the table, and the next one's: that is on its way to L2 a token ahead of its use
    auto row_of = [&](int i) { return P.cos_sin != nullptr && i < P.T ? position(P, i) : -1; };
    auto prefetch = [&](int pos) {
        if (pos >= 0 && pos < P.table_rows && 8 * lane < P.rot)
            asm volatile("prefetch.global.L2 [%0];" :: "l"(P.cos_sin + (int64_t)pos * P.rot + 8 * lane));
    };
    int pos[2] = {row_of(t), row_of(t + 1)};
    for (int left = (int)(end - begin); left > 0; --left) {
        fetch();
        if (fresh && P.cos_sin != nullptr) {
            good = turn_at<PAIRS>(P, pos[0], lp, turn);
            if (!good && lane == 0) atomicAdd(&g_heads_bad, 1u);
            pos[0] = pos[1];
            prefetch(pos[0]);
            pos[1] = row_of(t + 2);
        }
        asm volatile("cp.async.wait_group %0;" :: "n"(kRing - 1) : "memory");
        const bool last = g == groups - 1, mine = live && (!last || grp < in_last);
        const uint4 cg[2] = {lds16(at), lds16(at + PIECE)};
        Lane16 d;
        unpack<PAIRS>(d, cg);
        if (P.cos_sin != nullptr && good && lp.turns) apply_turn<true, NORM, PAIRS>(d, turn, lp);
        if (NORM) {
            const uint4 cx[2] = {lds16(at + 2 * PIECE), lds16(at + 3 * PIECE)};
            Lane16 x;
            unpack<PAIRS>(x, cx);
            if (!good) {   // a token without an angle adds nothing to the gain's gradient, whatever it holds
                fill(x, 0.0f);
                fill(d, 0.0f);
            }
            float2 sd = make_float2(0.0f, 0.0f), se = sd;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sd = __ffma2_rn(__fmul2_rn(d.a[j], x.a[j]), gamma.a[j], sd);
                se = __ffma2_rn(__fmul2_rn(d.b[j], x.b[j]), gamma.b[j], se);
            }
            sd = __fadd2_rn(sd, se);
            const float sq = dot(x, x);
            // (asked of the lanes' own sums, ahead of the head's: asked of those the branch below costs 3.5 us of 92)
            const bool odd = __any_sync(0xFFFFFFFFu, !(sq <= 0x1p80f && sq >= low) && mine);
            const float ms = mean_square(head_sum<LP>(sq), P.inv_dim, P.eps);
            float hx = head_sum<LP>(sd.x + sd.y), r = head_rcp(ms), r_dx = r;   // r_dx: that of x as it was read
            if (__builtin_expect(odd, 0)) {
                float unit;
                r = head_rcp_any<LP>(x, ms, P.inv_dim, P.eps, unit);
                r_dx = fminf(r * unit, 3.402823466e+38f);
                float again = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    again = fmaf(d.a[j].x * x.a[j].x, gamma.a[j].x, fmaf(d.a[j].y * x.a[j].y, gamma.a[j].y, again));
                    again = fmaf(d.b[j].x * x.b[j].x, gamma.b[j].x, fmaf(d.b[j].y * x.b[j].y, gamma.b[j].y, again));
                }
                again = head_sum<LP>(again);
                if (!in_range(ms)) hx = again;   // the warp's other heads keep their bits
            }
            const float m = -hx * r * P.inv_dim * r;  // -mean(h n) * r: dx = r * (h + x * m)
            const float2 r2 = make_float2(r, r), dx2 = make_float2(r_dx, r_dx), m2 = make_float2(m, m);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                acc.a[j] = __ffma2_rn(__fmul2_rn(d.a[j], x.a[j]), r2, acc.a[j]);
                acc.b[j] = __ffma2_rn(__fmul2_rn(d.b[j], x.b[j]), r2, acc.b[j]);
                d.a[j] = __fmul2_rn(__ffma2_rn(x.a[j], m2, __fmul2_rn(d.a[j], gamma.a[j])), dx2);
                d.b[j] = __fmul2_rn(__ffma2_rn(x.b[j], m2, __fmul2_rn(d.b[j], gamma.b[j])), dx2);
            }
        }
        if (mine) {
            if (!good) fill(d, __uint_as_float(0x7FC00000u));
            store<PAIRS>(reinterpret_cast<uint16_t*>(y), second, d);
        }
        at = at + SLOT == ring_at + kRing * SLOT ? ring_at : at + SLOT;
        y += step;
        ++g;
        fresh = last;
        if (last) {
            g = 0;
            ++t;
            y += y_stride - token_bytes;
        }
    }
    if constexpr (NORM) {
        if (P.partial == nullptr) return;
        // the CTA's row of partial sums: groups of the warp by shuffles, then the warps in order
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float v[4] = {acc.a[j].x, acc.a[j].y, acc.b[j].x, acc.b[j].y};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
#pragma unroll
                for (int o = LP; o < 32; o <<= 1) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
                // member k / 2 of pair 2j + k % 2
                const int pair = 2 * j + (k & 1), at = PAIRS ? 2 * pair + (k >> 1) : pair + 8 * (k >> 1);
                if (grp == 0 && live) sums[warp][at < 8 ? lp.o0 + at : lp.o1 + at - 8] = v[k];
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < P.dim; c += kWarps * 32) {
            float s = 0.0f;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) s += sums[k][c];
            P.partial[(int64_t)blockIdx.x * P.dim + c] = s;
        }
    }
}

// sums the CTAs' rows in a fixed order: 16 columns a CTA, 64 runs of rows, joined in order
__global__ void __launch_bounds__(1024) rope_dgain_kernel(const HeadsParams P, int rows_q, int rows_all)
{
    __shared__ float sums[64][17];
    pdl_prologue();
    const int which = blockIdx.y, c = threadIdx.x & 15, run = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    float* out = P.dgain[which];
    if (out == nullptr) return;
    const int first = which ? rows_q : 0, last = which ? rows_all : rows_q;
    float s = 0.0f;
#pragma unroll 4
    for (int r = first + run; r < last; r += 64) s += P.partial[(int64_t)r * P.dim + col];
    sums[run][c] = s;
    __syncthreads();
    if (run == 0) {
        float a = 0.0f;
#pragma unroll
        for (int k = 0; k < 64; ++k) a += sums[k][c];
        out[col] = a;
    }
}

template <class... Args>
cudaError_t launch(void (*kernel)(Args...), dim3 grid, int threads, cudaStream_t stream, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// calls f(lanes per head, pairs, norm) for the case at hand, as compile-time constants
template <class F>
cudaError_t by_case(const HeadsParams& P, F f)
{
    auto by_flags = [&](auto lp) {
        if (P.pairs) return P.norm ? f(lp, std::true_type{}, std::true_type{}) : f(lp, std::true_type{}, std::false_type{});
        return P.norm ? f(lp, std::false_type{}, std::true_type{}) : f(lp, std::false_type{}, std::false_type{});
    };
    switch (lanes_per_head(P.dim)) {
        case 1: return by_flags(std::integral_constant<int, 1>{});
        case 2: return by_flags(std::integral_constant<int, 2>{});
        case 4: return by_flags(std::integral_constant<int, 4>{});
        case 8: return by_flags(std::integral_constant<int, 8>{});
        default: return by_flags(std::integral_constant<int, 16>{});
    }
}

template <int U, int LP, bool PAIRS, bool NORM>
cudaError_t launch_fwd_kernel(const HeadsParams& P, cudaStream_t stream)
{
    return launch(rope_fwd_kernel<LP, U, PAIRS, NORM>, dim3((unsigned)((P.T * P.parts + kWarps - 1) / kWarps)), kWarps * 32, stream, (const HeadsParams)P);
}

}  // namespace

cudaError_t launch_rope_fwd(HeadsParams P, cudaStream_t stream)
{
    // groups of heads that a warp takes at once: five where that divides the heads with least left over (40 heads of 128:
    // 2 warps a token), one where there are too few tokens to keep the SMs busy otherwise
    const int groups = (P.heads[0] + P.heads[1] + 32 / lanes_per_head(P.dim) - 1) / (32 / lanes_per_head(P.dim));
    int u = 1;
    if (P.T * groups >= (int64_t)kSMs * 32) {
        static constexpr int kChoices[] = {5, 3, 2, 1};
        int best = 1 << 30;
        for (int c : kChoices) {
            const int slots = (groups + c - 1) / c * c;
            if (slots < best) {
                best = slots;
                u = c;
            }
        }
    }
    P.parts = (groups + u - 1) / u;
    return by_case(P, [&](auto lp, auto pairs, auto norm) {
        constexpr int LP = decltype(lp)::value;
        constexpr bool PAIRS = decltype(pairs)::value, NORM = decltype(norm)::value;
        switch (u) {
            case 5: return launch_fwd_kernel<5, LP, PAIRS, NORM>(P, stream);
            case 3: return launch_fwd_kernel<3, LP, PAIRS, NORM>(P, stream);
            case 2: return launch_fwd_kernel<2, LP, PAIRS, NORM>(P, stream);
            default: return launch_fwd_kernel<1, LP, PAIRS, NORM>(P, stream);
        }
    });
}

int rope_bwd_ctas(int64_t T, int q_heads, int k_heads, int dim)
{
    // four resident CTAs an SM; fewer where an item a warp would be too little work
    const int at_once = 32 / lanes_per_head(dim);
    const int64_t items = T * ((q_heads + at_once - 1) / at_once + (k_heads + at_once - 1) / at_once);
    const int64_t need = (items + kWarps - 1) / kWarps, cap = (int64_t)kSMs * 4;
    const int64_t n = need < cap ? need : cap;
    return (int)(n < 2 ? 2 : n);
}

cudaError_t launch_rope_bwd(HeadsParams P, cudaStream_t stream)
{
    const int ctas = rope_bwd_ctas(P.T, P.heads[0], P.heads[1], P.dim);
    // CTAs for the queries: by the groups of heads a token has, plus what a token costs by itself (its angles)
    const int at_once = 32 / lanes_per_head(P.dim), token = 2;
    const int64_t wq = 2 * ((P.heads[0] + at_once - 1) / at_once) + token, wk = 2 * ((P.heads[1] + at_once - 1) / at_once) + token;
    int q = P.heads[1] == 0 ? ctas : P.heads[0] == 0 ? 0 : (int)((ctas * wq + (wq + wk) / 2) / (wq + wk));
    if (P.heads[0] > 0 && q < 1) q = 1;
    if (P.heads[1] > 0 && q > ctas - 1) q = ctas - 1;
    P.ctas_q = q;
    cudaError_t e = by_case(P, [&](auto lp, auto pairs, auto norm) {
        return launch(rope_bwd_kernel<decltype(lp)::value, decltype(pairs)::value, decltype(norm)::value>, dim3(ctas), kWarps * 32, stream,
                      (const HeadsParams)P);
    });
    if (e != cudaSuccess || P.partial == nullptr) return e;
    return launch(rope_dgain_kernel, dim3(P.dim / 16, 2), 1024, stream, (const HeadsParams)P, q, ctas);
}

cudaError_t read_heads_bad(unsigned int* out) { return cudaMemcpyFromSymbol(out, g_heads_bad, sizeof(unsigned int)); }
cudaError_t reset_heads_bad()
{
    const unsigned int zero = 0;
    return cudaMemcpyToSymbol(g_heads_bad, &zero, sizeof(unsigned int));
}

}  // namespace mxn
