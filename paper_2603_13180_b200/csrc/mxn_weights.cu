// Summed attention weights of the keys of the paged 8-bit cache: what each key has been given by all queries of a call.
//
//   w_t = earlier_t + sum over rows i of exp(scale q_i . k_t - lse_i),   k_t = 2^(sk - 127) * code
//
// over the rows of t's sequence that see t and the query heads that share the key head; lse is the attention's logarithm of the sum.
// Every key's sum stands by itself, so that no two warps meet in one and nothing is joined.
//
// Few rows (up to kRows a sequence and key head): bound by HBM, dim bytes of codes, 4 (and 4 earlier) of sums a token and head.  A warp
// takes tiles of 32 tokens.  The order of the dimensions within a product is free: a thread reads one run of dim / 4 bytes of each of
// its four tokens straight into registers, in which the codes become f16 operands (exact), and asks for the next tile's over them once the
// products have read them.  q is scaled by a power of two that brings its row's largest to [2^14, 2^15): f16 holds a bf16 value exactly but
// for elements below 2^-28 of that.  The power is at most 2^110, by which f16 still holds the smallest bf16 (2^-133 times it is 2^-23): the factor that
// takes it back, with the scores' scale, then stays a normal number for scales down to 2^-16.
//
// Measured, 32 query and 8 key heads of 128, 64 sequences of up to 8192 keys, one token each, added to earlier sums: 70 us, 5.1 TB/s, 0.79
// of a copy's rate.  Two sets of registers and four CTAs an SM took 94 us, one set and five 74, with fewer instructions beside the products 70 (some 490 a
// tile now, of which 145 are products, conversions and exponentials: half of the issue slots).  A ring of tiles filled by the tensor copy
// engine took 73 with two stages a warp and 80 with three (fewer warps fit beside more shared memory), six CTAs an SM 78 (spills).
#include "mxn_attn.cuh"

namespace mxn {

namespace {

constexpr int kWarps = 4, kTile = 32, kRows = 64;
constexpr float kLog2e = 1.4426950408889634f;

__device__ unsigned int g_weights_bad = 0;   // pages out of range within a sequence's length

__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// FEW: up to eight rows, whose operands stay in registers; else up to kRows, in shared memory
template <int DIM, bool FEW>
__global__ void __launch_bounds__(kWarps * 32, FEW ? 5 : 4) key_weights_kernel(const WeightsParams W)
{
    constexpr int KS = DIM / 16;
    __shared__ uint2 q_frag[FEW ? 1 : kRows / 8][FEW ? 1 : KS][FEW ? 1 : 32];
    __shared__ float2 q_row[FEW ? 1 : kRows];   // factor of the scores, -lse in powers of two
    __shared__ int2 q_see[FEW ? 1 : kRows];     // first and past the last key seen (but for the first `sinks`)
    pdl_prologue();
    const AttnParams& P = W.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    uint32_t b = blockIdx.x;
    const int split = (int)(b % (uint32_t)P.splits);
    b /= (uint32_t)P.splits;
    const int h = (int)(b % (uint32_t)P.kv_heads), seq = (int)(b / (uint32_t)P.kv_heads);
    const AttnSequence S = attn_sequence(P, seq);
    const int G = P.group, rows = S.nq * G, end = S.len;
    const int k0 = (int)min((int64_t)end, (int64_t)split * P.chunk), k1 = (int)min((int64_t)end, (int64_t)k0 + P.chunk);
    if (k0 >= k1) return;
    const int tiles = (k1 - k0 + kTile - 1) / kTile, mine = tiles > warp ? (tiles - warp + kWarps - 1) / kWarps : 0;
    const int32_t* const table = P.page_table + (int64_t)seq * P.max_pages;
    const int per_page = P.page_shift - P.block_shift;
    const bool wide = (reinterpret_cast<uintptr_t>(P.k_codes) & 31u) == 0u;   // (codes are promised to be 16-byte aligned)
    const int old_end = W.earlier == nullptr ? 0 : S.nq > 0 ? min(S.shift, k1) : k1;   // tokens in front of the call's own have sums from earlier
    // keys that any row sees: [lo, hi) and the first `sinks`
    const int pos0 = S.shift, pos1 = S.shift + S.nq - 1;
    const int lo = first_seen(pos0, P.window), hi = rows > 0 ? (P.causal ? min(pos1 + 1, end) : end) : 0, sinks = min(P.sinks, hi);
    auto tile_at = [&](int i) { return k0 + (warp + i * kWarps) * kTile; };
    auto page_at = [&](int i) -> int {   // page of this half warp's run of 16 tokens
        const int t = tile_at(i) + (lane & 16);
        return i < mine && t < k1 ? __ldg(table + (t >> P.page_shift)) : -1;
    };

    // ---- a tile on its way: codes of tokens g, 8 + g, 16 + g, 24 + g, dimensions c * DIM/4 on; what its sums need ----
    uint4 w[4][DIM / 64];
    uint32_t scale;      // of this half warp's run of 16 tokens
    int64_t at;          // of the sum that this thread writes, -1: of none
    float earlier;
    bool bad = false;
    const int page_mask = P.page - 1, out_token = 16 * (c >> 1) + 8 * (c & 1) + g;   // the token of a tile whose sum this thread writes
    auto seen = [&](int t0) { return (t0 < hi && t0 + kTile > lo) || t0 < sinks; };
    auto load = [&](int i, int pg) {   // by a whole warp; pg = page_at(i)
        const int t0 = tile_at(i), run = t0 + (lane & 16);
        const bool wanted = i < mine && run < k1;
        bad |= wanted && (uint32_t)pg >= (uint32_t)P.num_pages;
        const int tile = wanted && (uint32_t)pg < (uint32_t)P.num_pages ? pg * P.kv_heads + h : -1;   // (fewer than 2^31)
        scale = tile >= 0 ? __ldg(P.k_scales + ((int64_t)tile << per_page) + ((run & page_mask) >> P.block_shift)) : 0u;
        const int out_tile = __shfl_sync(0xFFFFFFFFu, tile, 8 * (c & 2)), place = t0 + out_token;
        at = out_tile >= 0 && place < k1 ? ((int64_t)out_tile << P.page_shift) + (place & page_mask) : -1;
        earlier = at >= 0 && place < old_end ? W.earlier[at] : 0.0f;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int from = __shfl_sync(0xFFFFFFFFu, tile, 16 * t);
            const uint8_t* const p0 = P.k_codes + (((int64_t)from << P.page_shift) + ((t0 + 16 * t) & page_mask) + g) * DIM + c * (DIM / 4);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                uint4* const y = w[2 * t + x];
                const uint8_t* const p = p0 + 8 * x * DIM;
#pragma unroll
                for (int e = 0; e < DIM / 64; ++e) y[e] = make_uint4(0u, 0u, 0u, 0u);
                if (from >= 0 && t0 + 16 * t + 8 * x + g < k1 && seen(t0)) {
                    if (DIM == 128 && wide) {
                        uint32_t v[8];
                        ld_v8(p, v);
#pragma unroll
                        for (int e = 0; e < DIM / 64; ++e) y[e] = make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
                    } else {
#pragma unroll
                        for (int e = 0; e < DIM / 64; ++e) y[e] = __ldg(reinterpret_cast<const uint4*>(p) + e);
                    }
                }
            }
        }
    };
    int pg = page_at(0);
    load(0, pg);
    pg = page_at(1);

    // ---- the rows: eight at a time by a warp; thread (g, c) reads a quarter of row g ----
    uint32_t qb[KS][2];
    float2 my_row = make_float2(0.0f, 0.0f);
    int2 my_see = make_int2(0, 0);
    auto prepare = [&](int eight) {
        const int row = 8 * eight + g, qt = P.by_group(row);
        const bool live = row < rows;
        uint4 raw[DIM / 32];
        const int64_t head = (int64_t)h * G + row - (int64_t)qt * G, tok = (int64_t)S.q0 + qt;
        const uint16_t* qp = P.q + tok * P.q_stride + head * DIM + c * (DIM / 4);
#pragma unroll
        for (int i = 0; i < DIM / 32; ++i) raw[i] = live ? __ldg(reinterpret_cast<const uint4*>(qp) + i) : make_uint4(0, 0, 0, 0);
        const float lse = live ? __ldg(W.lse + tok * P.q_heads + head) : -INFINITY;
        const uint32_t* u = reinterpret_cast<const uint32_t*>(raw);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < DIM / 8; ++i) m = absmax_bf16x2(m, u[i]);
        float top = hmax_abs_to_f32(m);
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        const uint32_t E = __float_as_uint(top) >> 23, Ec = min(max(E, 31u), 254u);
        const float up = E == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float((268u - Ec) << 23);   // an infinity or NaN: NaN
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            qb[k][0] = pack_f16(bf16_lo(u[2 * k]) * up, bf16_hi(u[2 * k]) * up);
            qb[k][1] = pack_f16(bf16_lo(u[2 * k + 1]) * up, bf16_hi(u[2 * k + 1]) * up);
        }
        my_row = make_float2(P.scale * kLog2e * __uint_as_float((Ec - 14u) << 23), -lse * kLog2e);
        const int pos = S.shift + qt;
        // a row that the attention found to see nothing gives nothing
        my_see = live && lse != -INFINITY ? make_int2(first_seen(pos, P.window), P.causal ? min(pos + 1, end) : end) : make_int2(0, 0);
    };
    float2 col_row[2];
    int2 col_see[2];
    if constexpr (FEW) {
        prepare(0);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int from = 8 * c + 4 * e;
            col_row[e] = make_float2(__shfl_sync(0xFFFFFFFFu, my_row.x, from), __shfl_sync(0xFFFFFFFFu, my_row.y, from));
            col_see[e] = make_int2(__shfl_sync(0xFFFFFFFFu, my_see.x, from), __shfl_sync(0xFFFFFFFFu, my_see.y, from));
        }
    } else {
        for (int eight = warp; 8 * eight < rows; eight += kWarps) {
            prepare(eight);
#pragma unroll
            for (int k = 0; k < KS; ++k) q_frag[eight][k][lane] = make_uint2(qb[k][0], qb[k][1]);
            if (c == 0) {
                q_row[8 * eight + g] = my_row;
                q_see[8 * eight + g] = my_see;
            }
        }
        __syncthreads();
    }

    for (int i = 0; i < mine; ++i) {
        const int t0 = tile_at(i), pg_next = page_at(i + 2);
        const bool any = seen(t0);
        const float kf[2] = {e8m0_to_f32(__shfl_sync(0xFFFFFFFFu, scale, 0)), e8m0_to_f32(__shfl_sync(0xFFFFFFFFu, scale, 16))};
        const int64_t out = at;
        const float before = earlier;
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};   // tokens g, 8 + g, 16 + g, 24 + g; this thread's columns
        float s[2][4];
        auto scores = [&](const uint2* frag) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[t][e] = 0.0f;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    uint32_t a0, a1, a2, a3;
                    widen(word(w[2 * t][k / 4], k % 4), a0, a2);
                    widen(word(w[2 * t + 1][k / 4], k % 4), a1, a3);
                    const uint2 f = FEW ? make_uint2(qb[k][0], qb[k][1]) : frag[k * 32];
                    mma_f16(s[t], a0, a1, a2, a3, f.x, f.y);
                }
            }
        };
        auto add = [&](const float2 (&cr)[2], const int2 (&cs)[2]) {
            if (__all_sync(0xFFFFFFFFu, t0 >= max(cs[0].x, cs[1].x) && t0 + kTile <= min(cs[0].y, cs[1].y))) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[2 * t + (e >> 1)] += ex2(fmaf(s[t][e], kf[t] * cr[e & 1].x, cr[e & 1].y));
            } else {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = ex2(fmaf(s[t][e], kf[t] * cr[e & 1].x, cr[e & 1].y));
                        const int place = t0 + 16 * t + 8 * (e >> 1) + g;
                        sum[2 * t + (e >> 1)] += place < cs[e & 1].y && (place >= cs[e & 1].x || place < sinks) ? p : 0.0f;
                    }
            }
        };
        if constexpr (FEW) {
            scores(nullptr);
            load(i + 1, pg);   // over the codes at hand: more warps hide more than a second set of registers did
            if (any) add(col_row, col_see);
        } else {
            if (any)
                for (int y = 0; 8 * y < rows; ++y) {
                    float2 cr[2];
                    int2 cs[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        cr[e] = q_row[8 * y + 2 * c + e];
                        cs[e] = q_see[8 * y + 2 * c + e];
                    }
                    scores(&q_frag[y][0][lane]);
                    add(cr, cs);
                }
            load(i + 1, pg);
        }
        pg = pg_next;
        // over the four threads of a token's columns; thread c keeps sum[c]
        const bool up = c & 2, odd = c & 1;
        const float a0 = (up ? sum[2] : sum[0]) + __shfl_xor_sync(0xFFFFFFFFu, up ? sum[0] : sum[2], 2);
        const float a1 = (up ? sum[3] : sum[1]) + __shfl_xor_sync(0xFFFFFFFFu, up ? sum[1] : sum[3], 2);
        const float all = (odd ? a1 : a0) + __shfl_xor_sync(0xFFFFFFFFu, odd ? a0 : a1, 1);
        if (out >= 0) W.sums[out] = before + all;
    }
    if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) atomicAdd(&g_weights_bad, 1u);
}

template <class K>
cudaError_t launch(K kernel, int64_t ctas, cudaStream_t stream, const WeightsParams& W)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kWarps * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, W);
}

}  // namespace

int64_t plan_weights(WeightsParams& W)
{
    AttnParams& P = W.a;
    W.many = (int64_t)P.max_q * P.group > kRows;
    if (W.many) {
        // query tiles of up to 128 rows: whole tokens, or one token's heads in parts
        W.tile_heads = P.group < 128 ? P.group : 128;
        W.tile_tokens = 128 / W.tile_heads < P.n ? 128 / W.tile_heads : (int)P.n;
        W.head_parts = (int)ceil_div(P.group, W.tile_heads);
        // CTAs for a key tile: more while the SMs are not filled twice and each still has four query tiles
        const int64_t units = ceil_div(P.max_len, 256) * P.seqs * P.kv_heads, tiles = ceil_div(P.max_q, W.tile_tokens) * W.head_parts;
        W.ranks = 1;
        while (W.ranks < 8 && units * W.ranks < 2 * kSMs && tiles >= 8 * W.ranks) W.ranks *= 2;
        return units * W.ranks;
    }
    // Chunks of 32 tiles (eight for each warp), or of one tile for each warp where CTAs would be fewer than three an SM; nothing is joined,
    // so a chunk costs no more than its start.
    const int64_t units = (int64_t)P.seqs * P.kv_heads, least = kWarps * kTile;
    P.chunk = 8 * least;
    if (units * ceil_div(P.max_len, P.chunk) < 3 * kSMs) P.chunk = least;
    P.splits = (int)ceil_div(P.max_len, P.chunk);
    return units * P.splits;
}

cudaError_t launch_weights(const WeightsParams& W, int64_t ctas, cudaStream_t stream)
{
    const AttnParams& P = W.a;
    if (W.many) return launch_weights_many(W, ctas, stream);
    const bool few = (int64_t)P.max_q * P.group <= 8;
    if (P.dim == 128) return few ? launch(key_weights_kernel<128, true>, ctas, stream, W) : launch(key_weights_kernel<128, false>, ctas, stream, W);
    return few ? launch(key_weights_kernel<64, true>, ctas, stream, W) : launch(key_weights_kernel<64, false>, ctas, stream, W);
}

cudaError_t read_weights_counters(unsigned int* timeouts, unsigned int* bad)
{
    unsigned int more = 0;
    cudaError_t e = cudaMemcpyFromSymbol(bad, g_weights_bad, sizeof(unsigned int));
    if (e == cudaSuccess) e = read_weights_many_counters(timeouts, &more);
    *bad += more;
    return e;
}
cudaError_t reset_weights_counters(bool timeouts)
{
    const unsigned int zero = 0;
    const cudaError_t e = timeouts ? cudaSuccess : cudaMemcpyToSymbol(g_weights_bad, &zero, sizeof(unsigned int));
    return e != cudaSuccess ? e : reset_weights_many_counters(timeouts);
}

}  // namespace mxn
