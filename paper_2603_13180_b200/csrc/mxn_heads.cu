// RMS norm of every query and key head with the position rotation in the same pass, and its gradient.
//
//   n = x * r,  r = 1 / sqrt(mean x^2 + eps) over the head;  u = n * gamma;  y = R(position) u
//   du = R^T dy;  dgamma = sum over tokens and heads of du * n;  h = du * gamma;  dx = r * (h - n * mean(h * n))
//
// Both are bound by HBM: 4 bytes an element forward (read x, write y), 6 backward (x, dy, dx).  A head of `dim` elements is
// held by dim/16 lanes (see mxn_rope.cuh), so the head's sums take log2(dim/16) shuffles and the rotation none; a warp
// works on 32*16/dim heads at a time and keeps the token's cosines and sines in registers over all of its heads.
// The gradient recomputes r from x, which it reads anyway, instead of loading a saved one.
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
__device__ __forceinline__ void st16(uint16_t* p, const float* x)
{
    const uint32_t r[4] = {pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
    st_v4(p, r);
}
template <int LP>
__device__ __forceinline__ float head_sum(float v)
{
#pragma unroll
    for (int o = LP / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
// 1 / sqrt(mean + eps); 0 for a head of zeros without eps, which then stays zero
__device__ __forceinline__ float head_rcp(float sum_sq, float inv_dim, float eps)
{
    const float ms = fmaf(sum_sq, inv_dim, eps);
    return ms > 0.0f ? rsqrtf(ms) : 0.0f;
}

// false: the token's position lies outside the table
__device__ __forceinline__ bool token_turn(const HeadsParams& P, int64_t t, int sub, const LanePairs& lp, Turn& turn)
{
    if (P.cos_sin == nullptr) return true;
    const int64_t pos = P.positions != nullptr ? (int64_t)__ldg(P.positions + t) : t;
    if (pos < 0 || pos >= P.table_rows) return false;
    if (lp.turns) load_turn(turn, P.cos_sin + pos * P.rot, sub, P.rot);
    return true;
}

template <int LP, bool PAIRS, bool NORM>
__global__ void __launch_bounds__(kWarps * 32) rope_fwd_kernel(const HeadsParams P)
{
    constexpr int G = 32 / LP;   // heads a warp holds at a time
    constexpr int U = 2;         // ... twice, to have more loads in flight
    pdl_prologue();
    const int lane = threadIdx.x & 31, sub = lane % LP, grp = lane / LP;
    const int64_t w = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    const int64_t t = w / P.parts;
    if (t >= P.T) return;
    const int part = (int)(w - t * P.parts);
    const int heads = P.heads[0] + P.heads[1];
    const int begin = part * P.per_part, end = min(heads, begin + P.per_part);
    const bool live = 16 * sub < P.dim;
    const LanePairs lp = lane_pairs(live ? sub : 0, P.rot, PAIRS);
    Turn turn;
    const bool good = token_turn(P, t, sub, lp, turn);
    if (!good && lane == 0 && part == 0) atomicAdd(&g_heads_bad, 1u);

    for (int h0 = begin + grp; h0 - grp < end; h0 += G * U) {
        uint4 raw[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * G;
            raw[u][0] = raw[u][1] = make_uint4(0u, 0u, 0u, 0u);
            if (live && h < end) {
                const int which = h >= P.heads[0];
                const uint16_t* x = P.x[which] + t * P.x_stride[which] + (int64_t)(h - (which ? P.heads[0] : 0)) * P.dim;
                raw[u][0] = ld16(x + lp.o0);
                raw[u][1] = ld16(x + lp.o1);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * G;
            const int which = h >= P.heads[0];
            float x[16];
            unpack8(x, raw[u][0]);
            unpack8(x + 8, raw[u][1]);
            if (NORM) {
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) s = fmaf(x[i], x[i], s);
                const float r = head_rcp(head_sum<LP>(s), P.inv_dim, P.eps);
                const uint16_t* gain = P.gain[which];
                if (gain != nullptr && live) {
                    float g[16];
                    unpack8(g, __ldg(reinterpret_cast<const uint4*>(gain + lp.o0)));
                    unpack8(g + 8, __ldg(reinterpret_cast<const uint4*>(gain + lp.o1)));
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = x[i] * r * g[i];
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] *= r;
                }
            }
            if (P.cos_sin != nullptr) {
                if (!good) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(0x7FC00000u);   // loud: no angle for this token
                } else if (lp.turns) {
                    apply_turn<PAIRS, false>(x, turn);
                }
            }
            if (live && h < end) {
                uint16_t* y = P.y[which] + t * P.y_stride[which] + (int64_t)(h - (which ? P.heads[0] : 0)) * P.dim;
                st16(y + lp.o0, x);
                st16(y + lp.o1, x + 8);
            }
        }
    }
}

// One CTA works for the queries or for the keys only (the CTAs are shared out by their head counts), so that a lane carries
// 16 sums of one gain's gradient.  A warp walks over a contiguous run of (token, group of heads) items and asks for the next
// item's x and dy before it works on the present one.
template <int LP, bool PAIRS, bool NORM>
__global__ void __launch_bounds__(kWarps * 32, 4) rope_bwd_kernel(const HeadsParams P)
{
    constexpr int G = 32 / LP;
    __shared__ float sums[kWarps][256];
    pdl_prologue();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % LP, grp = lane / LP;
    const int which = (int)blockIdx.x >= P.ctas_q;
    const int64_t cta = which ? (int)blockIdx.x - P.ctas_q : (int)blockIdx.x, ctas = which ? (int)gridDim.x - P.ctas_q : P.ctas_q;
    const int heads = P.heads[which], groups = (heads + G - 1) / G;
    const int64_t items = P.T * groups, warps = ctas * kWarps, w = cta * kWarps + warp;
    const int64_t begin = items * w / warps, end = items * (w + 1) / warps;
    const bool live = 16 * sub < P.dim;
    const LanePairs lp = lane_pairs(live ? sub : 0, P.rot, PAIRS);
    const uint16_t* const x_base = P.x[which];
    const uint16_t* const g_base = P.grad[which];
    float acc[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
    uint4 gain[2];   // bf16 pairs
    gain[0] = gain[1] = make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);   // ones
    if (NORM && P.gain[which] != nullptr && live) {
        gain[0] = __ldg(reinterpret_cast<const uint4*>(P.gain[which] + lp.o0));
        gain[1] = __ldg(reinterpret_cast<const uint4*>(P.gain[which] + lp.o1));
    }
    Turn turn;
    bool good = true;
    int64_t t = begin / groups;
    int g = (int)(begin - t * groups);
    int64_t turn_of = -1;

    uint4 nx[2], ng[2];
    auto fetch = [&](int64_t tt, int gg) {
        const int h = gg * G + grp;
        nx[0] = nx[1] = ng[0] = ng[1] = make_uint4(0u, 0u, 0u, 0u);
        if (live && h < heads) {
            if (NORM) {
                const uint16_t* x = x_base + tt * P.x_stride[which] + (int64_t)h * P.dim;
                nx[0] = ld16(x + lp.o0);
                nx[1] = ld16(x + lp.o1);
            }
            const uint16_t* d = g_base + tt * P.grad_stride[which] + (int64_t)h * P.dim;
            ng[0] = ld16(d + lp.o0);
            ng[1] = ld16(d + lp.o1);
        }
    };
    if (begin < end) fetch(t, g);
    for (int64_t i = begin; i < end; ++i) {
        uint4 cx[2] = {nx[0], nx[1]}, cg[2] = {ng[0], ng[1]};
        const int64_t ct = t;
        const int h = g * G + grp;
        if (++g == groups) {
            g = 0;
            ++t;
        }
        if (i + 1 < end) fetch(t, g);
        if (ct != turn_of) {
            good = token_turn(P, ct, sub, lp, turn);
            turn_of = ct;
            if (!good && lane == 0) atomicAdd(&g_heads_bad, 1u);
        }
        float d[16];
        unpack8(d, cg[0]);
        unpack8(d + 8, cg[1]);
        if (P.cos_sin != nullptr && good && lp.turns) apply_turn<PAIRS, true>(d, turn);
        if (NORM) {
            float x[16], gamma[16], ss = 0.0f, sd = 0.0f;
            unpack8(gamma, gain[0]);
            unpack8(gamma + 8, gain[1]);
            unpack8(x, cx[0]);
            unpack8(x + 8, cx[1]);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                ss = fmaf(x[j], x[j], ss);
                sd = fmaf(d[j] * gamma[j], x[j], sd);
            }
            ss = head_sum<LP>(ss);
            sd = head_sum<LP>(sd);
            const float r = head_rcp(ss, P.inv_dim, P.eps);
            const float m = sd * r * P.inv_dim * r;   // mean(h n) * r: dx = r * (h - x * m)
            const float rg = good ? r : 0.0f;         // a token without an angle adds nothing to the gain's gradient
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                acc[j] = fmaf(d[j], x[j] * rg, acc[j]);
                d[j] = r * (d[j] * gamma[j] - x[j] * m);
            }
        }
        if (live && h < heads) {
            if (!good) {
#pragma unroll
                for (int j = 0; j < 16; ++j) d[j] = __uint_as_float(0x7FC00000u);
            }
            uint16_t* y = P.y[which] + ct * P.y_stride[which] + (int64_t)h * P.dim;
            st16(y + lp.o0, d);
            st16(y + lp.o1, d + 8);
        }
    }
    if constexpr (NORM) {
        if (P.partial == nullptr) return;
        // the CTA's row of partial sums: groups of the warp by shuffles, then the warps in order
#pragma unroll
        for (int o = LP; o < 32; o <<= 1)
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[j] += __shfl_xor_sync(0xFFFFFFFFu, acc[j], o);
        if (grp == 0 && live) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                sums[warp][lp.o0 + j] = acc[j];
                sums[warp][lp.o1 + j] = acc[8 + j];
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

// calls f.template operator()<LP, PAIRS, NORM>() for the case at hand
template <class F>
cudaError_t by_case(const HeadsParams& P, F f)
{
    auto by_flags = [&](auto lp) {
        constexpr int LP = decltype(lp)::value;
        if (P.pairs) return P.norm ? f(std::integral_constant<int, LP>{}, std::true_type{}, std::true_type{})
                                   : f(std::integral_constant<int, LP>{}, std::true_type{}, std::false_type{});
        return P.norm ? f(std::integral_constant<int, LP>{}, std::false_type{}, std::true_type{})
                      : f(std::integral_constant<int, LP>{}, std::false_type{}, std::false_type{});
    };
    switch (lanes_per_head(P.dim)) {
        case 1: return by_flags(std::integral_constant<int, 1>{});
        case 2: return by_flags(std::integral_constant<int, 2>{});
        case 4: return by_flags(std::integral_constant<int, 4>{});
        case 8: return by_flags(std::integral_constant<int, 8>{});
        default: return by_flags(std::integral_constant<int, 16>{});
    }
}

}  // namespace

cudaError_t launch_rope_fwd(HeadsParams P, cudaStream_t stream)
{
    const int heads = P.heads[0] + P.heads[1], at_once = 32 / lanes_per_head(P.dim);
    // a warp takes all heads of a token, unless that would leave SMs without work (few tokens): then the heads are
    // shared out among as many warps as it takes to reach about four a scheduler
    const int most = (heads + at_once - 1) / at_once;
    const int64_t want = ((int64_t)kSMs * 16 + P.T - 1) / P.T;
    P.parts = (int)(want < 1 ? 1 : want > most ? most : want);
    P.per_part = ((most + P.parts - 1) / P.parts) * at_once;
    P.parts = (heads + P.per_part - 1) / P.per_part;
    const int64_t ctas = (P.T * P.parts + kWarps - 1) / kWarps;
    return by_case(P, [&](auto lp, auto pairs, auto norm) {
        return launch(rope_fwd_kernel<decltype(lp)::value, decltype(pairs)::value, decltype(norm)::value>, dim3((unsigned)ctas), kWarps * 32,
                      stream, (const HeadsParams)P);
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
    const int ctas = rope_bwd_ctas(P.T, P.heads[0], P.heads[1], P.dim), heads = P.heads[0] + P.heads[1];
    int q = (int)(((int64_t)ctas * P.heads[0] + heads / 2) / heads);
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
